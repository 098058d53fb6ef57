"""The scratch of the products of a linear layer in 8 bits, without a GPU: how much a call asks for, and what it does with as much as another one asked
for.  (The check of the size comes before the first CUDA call.)"""
import random

import pytest

import paper_2510_09103_b200 as A
from test_linear8_host import ENOWORKSPACE, OPS, _linear, _Scratch

HEAD = 16384           # more than the status words


def _ld(cols):
    return -(-cols // 16) * 16


def _desc(tokens, out, inn, **kw):
    return A.linear8_desc(tokens, out, inn, x8_ld=_ld(inn), w8_ld=_ld(inn), **kw)


SHAPES = [(14336, 4096), (2736, 1024), (12904, 304), (528, 80), (8, 8), (65536, 8), (8, 65536), (65536, 512), (4096, 4096), (1600, 6400), (512, 16384)]


@pytest.mark.parametrize("which", list(OPS))
@pytest.mark.parametrize("kind", [A.TYPE_BF16, A.TYPE_F32])
@pytest.mark.parametrize("out,inn", SHAPES)
def test_a_scratch_asked_for_with_some_tokens_does_for_fewer(which, kind, out, inn):
    rng = random.Random(out + inn)
    tokens = sorted({*range(1, 1200, 7), *(rng.randint(1, 20000) for _ in range(200)), 64, 128, 256, 512, 559, 768, 1024, 2048, 4096, 8192, 16384, 1 << 20, 1 << 24})
    form = dict(y_dtype=kind, dx_dtype=kind, dweight_dtype=kind)
    sizes = [A.adapm_linear8_scratch_bytes(_desc(t, out, inn, **form), which) for t in tokens]
    least = None
    for t, size in reversed(list(zip(tokens, sizes))):
        assert size > 0
        least = size if least is None else min(least, size)
        # far apart, so that no buffer lies over another
        at = {name: (i + 1) << 45 for i, name in enumerate(OPS[which])}
        code = _linear(which, _desc(t, out, inn, **form), out=9 << 45, scratch=_Scratch(least, 10 << 45), **at)
        assert code != ENOWORKSPACE, (t, size, least)


def test_calls_that_use_the_status_words_alone_ask_for_no_more():
    """One token, few tokens, and few tiles: by rows of the weight or by strips."""
    for kind in (A.TYPE_BF16, A.TYPE_F32):
        form = dict(y_dtype=kind, dx_dtype=kind, dweight_dtype=kind)
        for which in OPS:
            assert 0 < A.adapm_linear8_scratch_bytes(_desc(1, 4096, 4096, **form), which) <= HEAD or which == A.LINEAR8_WEIGHT_GRAD
            assert 0 < A.adapm_linear8_scratch_bytes(_desc(0, 4096, 4096, **form), which) <= HEAD
        for tokens in (1, 16, 64):
            assert A.adapm_linear8_scratch_bytes(_desc(tokens, 14336, 4096, **form), A.LINEAR8_INPUT_GRAD) <= HEAD
        assert A.adapm_linear8_scratch_bytes(_desc(777, 1376, 512, **form), A.LINEAR8_WEIGHT_GRAD) <= HEAD
        assert A.adapm_linear8_scratch_bytes(_desc(8192, 14336, 4096, **form), A.LINEAR8_FORWARD) <= HEAD
