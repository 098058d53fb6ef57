"""What dropout, the RMS norm and the head loss refuse and what they let through where buffers lie near one another, without a GPU:
a call whose arguments are in order ends at the first CUDA call, with an error of its own."""
import pytest

import paper_2510_09103_b200 as A
import test_operators_host as H
from test_operators_host import ECUDA, EINVAL, P, _Scratch, _dropout, _head, _head_grad, _norm, _norm_grad

pytestmark = pytest.mark.skipif(not H._no_device(), reason="addresses that stand for buffers are for a machine without a device")

# ---- matrices that lie between one another's rows ---------------------------------------------------------


@pytest.mark.parametrize("cols,ld,at,ok", [(16, 32, 32, True), (16, 32, 30, False), (16, 32, 34, False), (16, 40, 40, True), (16, 40, 48, True),
                                           (16, 40, 50, False), (16, 32, 0, False), (16, 32, -32, True), (16, 32, -30, False), (16, 48, 96 + 32, True),
                                           (16, 48, 96, False), (16, 32, 3 * 64 + 32, True), (16, 32, 3 * 64 + 30, False), (16, 32, 4 * 64, True)])
def test_rows_between_rows(cols, ld, at, ok):
    """Four rows of 32 bytes; an output `at` bytes from an input of the same pitch shares an element with it or does not."""
    want = ECUDA if ok or at == 0 else EINVAL
    assert _dropout(cols=cols, x_ld=ld, y_ld=ld, y=P + at) == want
    assert _dropout(cols=cols, x_ld=64, residual=2 * P, residual_ld=ld, y_ld=ld, x=9 * P, y=2 * P + at) == want
    desc = A.rmsnorm_desc(4, cols, x_ld=ld, y_ld=ld, sum_ld=ld, residual_ld=ld)
    assert _norm(desc, x=2 * P, weight=9 * P, y=2 * P + at) == want
    assert _norm(desc, x=2 * P, weight=9 * P, y=None, sum=2 * P + at) == want
    assert _norm(desc, x=5 * P, weight=9 * P, y=2 * P, sum=2 * P + at) == (ECUDA if ok else EINVAL)
    assert _norm_grad(desc, sum=12 * P, dresidual=12 * P + at) == want
    assert _norm_grad(desc, dx=12 * P + at, dresidual=12 * P) == (ECUDA if ok else EINVAL)


def test_other_pitches_and_types_over_one_another_are_refused():
    assert _dropout(x_ld=32, y_ld=48, y=P + 32) == EINVAL
    assert _norm(A.rmsnorm_desc(4, 64, x_ld=128, y8_ld=128), y8=P + 128, y8_scales=7 * P) == EINVAL
    # a pitch of 128 elements of two bytes and one of 256 elements of one byte are the same
    assert _norm(A.rmsnorm_desc(4, 64, x_ld=128, y8_ld=256), y8=P + 128, y8_scales=7 * P) == ECUDA
    assert _norm(A.rmsnorm_desc(4, 64, x_ld=128, y8_ld=256), y8=P + 126, y8_scales=7 * P) == EINVAL


@pytest.mark.parametrize("at,ok", [(128, True), (112, False), (160, False), (144, True), (-128, True), (-144, True), (-160, False), (3 * 272 + 128, True), (3 * 272 + 112, False)])
def test_head_gradients_between_rows(at, ok):
    """Rows of 128 bytes at a pitch of 272."""
    desc = A.head_loss_desc(4, 4, 64, hidden_ld=136, weight_ld=136)
    want = ECUDA if ok else EINVAL
    assert _head_grad(desc, dhidden=P + at, dweight=None) == want
    assert _head_grad(desc, dhidden=None, dweight=2 * P + at) == want
    assert _head_grad(desc, hidden=20 * P, dhidden=2 * P + at) == want
    assert _head_grad(desc, hidden=20 * P, weight=21 * P, dhidden=6 * P, dweight=6 * P + at) == want


# ---- vectors and scratch ----------------------------------------------------------------------------------

def test_dropout_over_its_step_word():
    assert _dropout(y=2 * P, step=2 * P + 8) == EINVAL and _dropout(y=2 * P, step=2 * P + 128) == ECUDA


def test_norm_vectors_over_matrices():
    desc = A.rmsnorm_desc(4, 64)
    for name in ("x", "residual", "sum", "y", "weight"):
        at = dict(x=10 * P, residual=11 * P, sum=12 * P, y=13 * P, weight=14 * P)
        end = at[name] + (4 if name != "weight" else 1) * 128
        assert _norm(desc, rstd=at[name] + 4, **at) == EINVAL, name
        assert _norm(desc, rstd=end, **at) == ECUDA, name
        assert _norm(desc, y8=20 * P, y8_scales=at[name] + 4, **at) == EINVAL, name
        assert _norm(desc, y8=20 * P, y8_scales=end, **at) == ECUDA, name
    assert _norm(desc, y8=20 * P, y8_scales=20 * P + 8) == EINVAL and _norm(desc, y8=20 * P, y8_scales=21 * P, rstd=21 * P + 12) == EINVAL
    assert _norm(desc, y8=20 * P, y8_scales=21 * P, rstd=21 * P + 16) == ECUDA and _norm(desc, y8=20 * P, y8_scales=21 * P, rstd=20 * P) == EINVAL
    for out in ("sum", "y"):
        assert _norm(A.rmsnorm_desc(4, 64, drop_p=0.1, step=30 * P), **{"y": None, out: 30 * P - 64}) == EINVAL
    # a vector between the rows of a matrix
    wide = A.rmsnorm_desc(4, 64, x_ld=128)
    assert _norm(wide, rstd=P + 128) == ECUDA and _norm(wide, rstd=P + 124) == EINVAL and _norm(wide, rstd=P + 244) == EINVAL
    assert _norm(wide, rstd=P + 3 * 256 + 128) == ECUDA and _norm(wide, rstd=P - 16) == ECUDA and _norm(wide, rstd=P - 12) == EINVAL


def test_norm_gradient_vectors_and_scratch_over_matrices():
    desc = A.rmsnorm_desc(4, 64, drop_p=0.1, step=30 * P)
    at = dict(dy=10 * P, dsum=11 * P, sum=12 * P, rstd=13 * P, weight=14 * P, dresidual=15 * P, dx=16 * P, dweight=17 * P)
    n = A.adapm_rmsnorm_backward_scratch_bytes(desc)
    assert _norm_grad(desc, scratch=_Scratch(n, 20 * P), **at) == ECUDA
    for name, where in at.items():
        assert _norm_grad(desc, scratch=_Scratch(n, where), **at) == EINVAL, name
        if name not in ("dresidual", "dx", "dweight"):
            assert _norm_grad(desc, scratch=_Scratch(n, 20 * P), **dict(at, dweight=where + 4)) == EINVAL, name
    assert _norm_grad(desc, scratch=_Scratch(n, 30 * P), **at) == EINVAL
    assert _norm_grad(desc, scratch=_Scratch(n, 20 * P), **dict(at, dweight=30 * P - 8)) == EINVAL
    assert _norm_grad(desc, scratch=_Scratch(n, 20 * P), **dict(at, dx=30 * P)) == EINVAL


def test_head_vectors_and_scratch_over_matrices():
    desc = A.head_loss_desc(4, 100, 64)
    n, m = A.adapm_head_loss_scratch_bytes(desc, False), A.adapm_head_loss_scratch_bytes(desc, True)
    at = dict(hidden=10 * P, weight=11 * P, targets=12 * P, loss=13 * P, lse=14 * P)
    assert _head(desc, scratch=_Scratch(n, 30 * P), **at) == ECUDA
    for name, where in at.items():
        assert _head(desc, scratch=_Scratch(n, where), **at) == EINVAL, name
        for vector in ("loss", "lse"):
            if name != vector:
                assert _head(desc, scratch=_Scratch(n, 30 * P), **dict(at, **{vector: where + 8})) == EINVAL, (name, vector)
    at = dict(hidden=10 * P, weight=11 * P, targets=12 * P, lse=14 * P, dloss=15 * P, dhidden=16 * P, dweight=17 * P)
    assert _head_grad(desc, scratch=_Scratch(m, 30 * P), **at) == ECUDA
    for name, where in at.items():
        assert _head_grad(desc, scratch=_Scratch(m, where), **at) == EINVAL, name
    # a larger buffer than the call needs may hold something else behind what it needs
    assert _head_grad(desc, scratch=_Scratch(1 << 40, 10 * P - m), **dict(at, hidden=10 * P)) == ECUDA
