"""What dropout, the RMS norm and the head loss refuse and what they let through where buffers lie near one another, without a GPU:
a call whose arguments are in order ends at the first CUDA call, with an error of its own."""
import pytest

import paper_2510_09103_b200 as A
import test_operators_host as H
from test_operators_host import ECUDA, EINVAL, P, _dropout, _head_grad, _norm, _norm_grad

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
