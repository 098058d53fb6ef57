"""What the linear layers in 8 bits refuse, and the tiles that their calls are cut into, without a GPU: every check of the arguments
comes before the first CUDA call, so it answers here as it does on a device."""
import ctypes as C
import os
import random
import subprocess

import pytest

import paper_2510_09103_b200 as A

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EALIGN, ERANGE, ENOWORKSPACE, EUNSUPPORTED = -1, -2, -3, -5, -6
P = 1 << 30            # an address that is never read: nothing is launched


def _code(f, *args):
    try:
        f(*args)
    except A.AdapmError as e:
        return e.code
    return 0


class _Scratch:
    """A buffer that says how long it is."""

    def __init__(self, n, at=16 * P):
        self.n, self.at = n, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 1


def _quant(d=None, back=False, **kw):
    d = d or A.quant8_desc(4, 64)
    a = dict(x=P, codes=2 * P, scales=3 * P)
    a.update(kw)
    if back:
        return _code(A.adapm_dequant8, d, a["codes"], a["scales"], a["x"], 0)
    return _code(A.adapm_quant8, d, a["x"], a["codes"], a["scales"], 0)


@pytest.mark.parametrize("back", [False, True])
def test_quant8_refusals(back):
    desc = A.quant8_desc
    q = lambda d=None, **kw: _quant(d, back, **kw)  # noqa: E731
    assert q(desc(-1, 64)) == EINVAL and q(desc(4, 0)) == EINVAL
    assert q(desc(1 << 31, 8)) == ERANGE and q(desc(1, (1 << 24) + 1)) == ERANGE
    assert q(desc(4, 64, dtype=2)) == EINVAL and q(desc(4, 64, code=2)) == EINVAL and q(desc(4, 64, group=64)) == EINVAL
    assert q(desc(4, 64, x_ld=63)) == EINVAL and q(desc(4, 64, codes_ld=63)) == EINVAL
    assert q(desc(1 << 30, 64, x_ld=1 << 40)) == ERANGE
    assert q(x=None) == EINVAL and q(codes=None) == EINVAL and q(scales=None) == EINVAL
    assert q(x=P + 1) == EALIGN and q(scales=3 * P + 2) == EALIGN
    assert q(codes=P) == EINVAL and q(codes=P + 64) == EINVAL and q(scales=P + 16) == EINVAL
    assert q(desc(4, 64, codes_ld=80), codes=P + 4 * 128 - 32) == EINVAL        # the last 32 bytes of x
    assert q(desc(0, 64), x=None) == 0
    if not back:
        assert q(scales=2 * P + 8) == EINVAL                                       # over the codes
        assert q(desc(4, 64, code=A.CODE_E4M3)) == EUNSUPPORTED
    lib = A.load()
    assert lib.adapm_quant8(None, P, 2 * P, 3 * P, 0) == EINVAL and lib.adapm_dequant8(None, P, 2 * P, 3 * P, 0) == EINVAL


OPS = {A.LINEAR8_FORWARD: ("x8", "xs", "w8", "ws"), A.LINEAR8_INPUT_GRAD: ("dy", "w8", "ws"), A.LINEAR8_WEIGHT_GRAD: ("dy", "x8", "xs")}
CALLS = {A.LINEAR8_FORWARD: "adapm_linear8_forward", A.LINEAR8_INPUT_GRAD: "adapm_linear8_input_grad", A.LINEAR8_WEIGHT_GRAD: "adapm_linear8_weight_grad"}


def _linear(which, d=None, out=9 * P, scratch=None, **kw):
    d = d or A.linear8_desc(24, 64, 96)
    a = {name: (i + 1) * P for i, name in enumerate(OPS[which])}
    a.update(kw)
    scratch = _Scratch(A.adapm_linear8_scratch_bytes(d, which) or 1024) if scratch is None else scratch
    return _code(getattr(A, CALLS[which]), d, *(a[name] for name in OPS[which]), out, scratch, 0)


@pytest.mark.parametrize("which", list(OPS))
def test_linear8_refusals(which):
    desc = A.linear8_desc
    r = lambda d=None, **kw: _linear(which, d, **kw)  # noqa: E731
    assert r(desc(-1, 64, 96)) == EINVAL and r(desc(4, 0, 96)) == EINVAL and r(desc(4, 64, 0)) == EINVAL
    assert r(desc((1 << 24) + 1, 64, 96)) == ERANGE and r(desc(4, (1 << 16) + 8, 96)) == ERANGE and r(desc(4, 64, (1 << 16) + 16)) == ERANGE
    assert r(desc(4, 60, 96, y_ld=64)) == EUNSUPPORTED and r(desc(4, 64, 100, x8_ld=112, w8_ld=112, dx_ld=104, dweight_ld=104)) == EUNSUPPORTED
    assert r(desc(4, 64, 96, y_dtype=2)) == EINVAL and r(desc(4, 64, 96, dx_dtype=-1)) == EINVAL and r(desc(4, 64, 96, dweight_dtype=7)) == EINVAL
    assert r(desc(4, 64, 96, x_code=2)) == EINVAL and r(desc(4, 64, 96, x_group=64)) == EINVAL
    assert r(desc(4, 64, 96, y_ld=56)) == EINVAL and r(desc(4, 64, 96, y_ld=68)) == EALIGN
    for name in OPS[which]:
        assert r(**{name: None}) == EINVAL, name
        at = (OPS[which].index(name) + 1) * P
        assert r(**{name: at + (2 if name in ("xs", "ws") else 8)}) == EALIGN, name
        assert r(out=at) == EINVAL, name                                            # the output over an input
        assert r(scratch=_Scratch(1 << 20, at)) == EINVAL, name                     # the scratch over an input
    assert r(out=None) == EINVAL and r(out=9 * P + 8) == EALIGN
    assert r(scratch=_Scratch(16)) == ENOWORKSPACE and r(scratch=_Scratch(1 << 20, 16 * P + 128)) == EALIGN
    assert r(scratch=_Scratch(1 << 20, 9 * P)) == EINVAL                            # the scratch over the output
    for field, used in (("x8_ld", "x8" in OPS[which]), ("w8_ld", "w8" in OPS[which]), ("dx_ld", which == A.LINEAR8_INPUT_GRAD), ("dweight_ld", which == A.LINEAR8_WEIGHT_GRAD)):
        if used:
            assert r(desc(4, 64, 96, **{field: 88})) == EINVAL and r(desc(4, 64, 96, **{field: 100})) == EALIGN, field
            assert r(desc(4, 64, 96, **{field: 1 << 31})) == ERANGE, field
    if which == A.LINEAR8_FORWARD:
        assert r(desc(4, 64, 96, x_code=A.CODE_E4M3)) == EUNSUPPORTED and r(desc(4, 64, 96, x_group=128)) == EUNSUPPORTED
        assert r(ws=4 * P + 4) == EALIGN
    if which == A.LINEAR8_WEIGHT_GRAD:
        assert r(desc(0, 64, 96, accumulate=True)) == 0 and r(desc(0, 64, 96), out=9 * P + 2) == EALIGN
    else:
        assert r(desc(0, 64, 96), out=None) == 0
    fn = getattr(A.load(), CALLS[which])
    assert fn(None, *[P] * len(OPS[which]), 9 * P, 16 * P, 4096, 0) == EINVAL
    assert A.load().adapm_linear8_scratch_bytes(None, which) == 0


def test_linear8_scratch_and_status_refusals():
    assert A.adapm_linear8_scratch_bytes(A.linear8_desc(4, 64, 96), 3) == 0 and A.adapm_linear8_scratch_bytes(A.linear8_desc(4, 63, 96), 1) == 0
    st = C.c_int32(0)
    assert A.load().adapm_linear8_status(None, 0, C.byref(st)) == EINVAL and A.load().adapm_linear8_status(P, 0, None) == EINVAL


# ---- the tiles of a call -----------------------------------------------------------------------------------

@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("linear8") / "plan.so")
    cuda = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2510_09103_b200", "csrc"),
                    "-I", cuda, "-o", path, os.path.join(ROOT, "tests", "linear8_plan_host.cpp")], check=True)
    lib = C.CDLL(path)
    lib.linear8_plan_wrong.restype = C.c_char_p
    return lib


def test_every_tile_and_part_once(plan):
    rng = random.Random(8)
    sizes = [(1, 8, 8), (1, 65536, 65536), (1 << 24, 8, 8), (256, 256, 256), (257, 264, 264), (65536, 512, 512), (65536, 64, 64), (4096, 4096, 4096), (1000, 2736, 1024)]
    spread = lambda hi: int(round(2 ** rng.uniform(0, hi)))  # noqa: E731
    sizes += [(spread(15), 8 * spread(12), 8 * spread(12)) for _ in range(300)]
    cut = 0
    for tokens, out, inn in sizes:
        d = A.linear8_desc(tokens, out, inn, x8_ld=-(-inn // 16) * 16, w8_ld=-(-inn // 16) * 16)
        for which in OPS:
            assert plan.linear8_plan_wrong(C.byref(d), which) is None, (tokens, out, inn, which, plan.linear8_plan_wrong(C.byref(d), which))
            cut += plan.linear8_parts(C.byref(d), which) > 1
    assert cut > 50
