"""How the head loss deals its tiles out to the pairs of CTAs, walked through on the host: every tile of the logits once, every part of
a gradient's long side once, nothing beside them, and no part that is not summed afterwards."""
import ctypes as C
import os
import random
import subprocess

import pytest

import paper_2510_09103_b200 as A

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_09103_b200", "csrc")
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")
BF16, F32 = A.TYPE_BF16, A.TYPE_F32


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("walk") / "walk.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                    "-I", os.path.join(CUDA, "include"), os.path.join(ROOT, "tests", "head_walk_host.cpp"), "-o", out], check=True)
    lib = C.CDLL(out)
    lib.head_walk_wrong.restype = C.c_char_p
    lib.head_walk_wrong.argtypes = [C.POINTER(A.adapm_head_loss)] + [C.c_int] * 5
    lib.head_pieces.argtypes = [C.POINTER(A.adapm_head_loss)]
    return lib


def _wrong(walk, tokens, vocab, hidden, dht=BF16, dwt=BF16, tv=None, backward=1, dh=1, dw=1, pairs=74):
    d = A.head_loss_desc(tokens, vocab, hidden, dhidden_dtype=dht, dweight_dtype=dwt)
    what = walk.head_walk_wrong(C.byref(d), backward, dh, dw, tokens if tv is None else tv, pairs)
    return what and (what.decode(), tokens, vocab, hidden, dht, dwt, tv, backward, dh, dw, pairs)


@pytest.mark.parametrize("tokens,vocab,hidden", [(100, 262208, 256), (100, 265792, 64), (70, 268864, 128), (256, 265768, 8)])
def test_a_last_piece_that_is_a_little_shorter_has_no_more_parts_than_are_summed(walk, tokens, vocab, hidden):
    assert _wrong(walk, tokens, vocab, hidden) is None


def test_last_pieces_of_every_length(walk):
    """Vocabularies just above one piece, in steps of a stage of K."""
    for tokens, dht in ((100, BF16), (64, BF16), (200, F32), (500, BF16)):
        for hidden in (8, 128, 256, 512):
            for vocab in range(262144, 262144 + 64 * 400, 64 * 7):
                assert _wrong(walk, tokens, vocab, hidden, dht) is None


def test_calls_of_all_sizes(walk):
    r = random.Random(1)

    def spread(a, b):
        return int(a * (b / a) ** r.random())

    for _ in range(1500):
        tokens, vocab, hidden = spread(1, 20000), spread(1, 140000), 8 * spread(1, 520)
        if tokens * vocab > 3e8:
            continue
        dh, dw = r.choice([(1, 1), (1, 1), (1, 0), (0, 1)])
        what = _wrong(walk, tokens, vocab, hidden, r.choice([BF16, F32]), r.choice([BF16, F32]), r.choice([None, None, 0, r.randint(0, tokens)]),
                      r.choice([1, 1, 1, 0]), dh, dw, r.choice([74, 74, r.randint(1, 74)]))
        assert what is None


def test_quotients_by_multiplication(walk):
    r = random.Random(2)
    for _ in range(20000):
        d, n = r.choice([r.randint(1, 40), r.randint(1, 1 << 20), 2 ** r.randint(0, 24)]), r.choice([r.randint(0, 2**31 - 1), 2**31 - 1])
        for k in (n, n // d * d, max(0, n // d * d - 1)):
            assert walk.head_quotient(k, d) == k // d
