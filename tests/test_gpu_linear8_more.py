"""Linear layers in 8 bits on a GPU: numbers at the edges of fp32's range, and the forms of their kernels that the sizes of test_gpu_linear8.py
pass by.  Helpers and derivations are those of that file."""
import pytest

import paper_2510_09103_b200 as A
import test_gpu_linear8 as T
from oracle import linear8_oracle as R
from test_gpu_operators import BF16, F32, HALF, _close, _rows, _tensor_sum

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---- codes next to half a step, of the smallest scales -----------------------------------------------------

@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("cols", [128, 127])
def test_codes_next_to_half_a_step_of_scales_whose_half_is_no_fp32_number(group, cols):
    """Scales from 2^-126 to 2^-125, in units of 2^-149: half of an odd one needs a bit that fp32 does not have there."""
    g = T._gen(11)
    rows = 4096
    unit = 2.0**-149
    s = torch.randint(1 << 23, 1 << 24, (rows,), generator=g, device="cuda").double()
    top = (127 * s * unit).float()                                      # its quotient by 127 is s or a neighbour
    s = (top.double() / 127).float().double() / unit
    assert (s == s.round()).all() and (s % 2 == 1).sum() > rows // 4
    codes = torch.randint(-126, 126, (rows, cols - 1), generator=g, device="cuda").double()
    at = (codes + 0.5) * s[:, None]                                     # half a step: a whole number of units, or half of one
    side = torch.randint(0, 2, (rows, cols - 1), generator=g, device="cuda").bool()
    x = torch.cat([top[:, None].double(), torch.where(side, at.floor(), at.ceil()) * unit], 1)
    # (a number of units above 2^24 is rounded to fp32: a neighbour of the middle all the same)
    codes, scales = T._check_quant(x.float(), "int8", group, False)
    assert torch.equal(scales.double(), s[:, None] * unit)


# ---- scales and gradients at the ends of the range -----------------------------------------------------------

def _far_apart(g, k, columns, pow2):
    """K numbers of dy and scales, one of them as small as the other is large, so that all of their products count; every seventh index of K with the largest
    dy that there are and scales above 1, whose codes are to be zero.  Signs of either kind."""
    power = torch.randint(-60, 61, (k,), generator=g, device="cuda").float()
    scales = torch.exp2(power) * (1 if pow2 else 1 + torch.rand(k, generator=g, device="cuda"))
    scales[3::5] = -scales[3::5]
    dy = torch.randn(k, columns, generator=g, device="cuda") * torch.exp2(-power)[:, None]
    empty = torch.zeros(k, dtype=torch.bool, device="cuda")
    empty[::7] = True
    dy[empty] = 3.3e38 * torch.sign(dy[empty])
    scales[empty] = 3 * torch.exp2(torch.randint(0, 60, (int(empty.sum()),), generator=g, device="cuda").float())
    if pow2:
        scales[empty] /= 3
    return dy.to(BF16), scales, empty


def _carried(size, want, k, dtype, columns):
    """Of terms that are carried with 24 bits (F32) or, with few columns, 16: two or three bf16 numbers to a term."""
    if dtype == F32:
        return T._bound(size, want, k, F32, False)
    assert columns <= 16
    return size * (_tensor_sum(2 * k, 256) + 2.0**-16) + want.abs() * HALF[BF16] * 1.01 + 1e-37


@pytest.mark.parametrize("pow2", [True, False])
@pytest.mark.parametrize("dtype,tokens,out,inn", [(BF16, 1, 520, 264), (BF16, 16, 2056, 136), (F32, 5, 520, 264), (F32, 70, 1032, 264), (F32, 1500, 2056, 1024)])
def test_input_grad_of_large_gradients_and_scales_far_apart(dtype, tokens, out, inn, pow2):
    g = T._gen(out + tokens)
    dy, ws, empty = _far_apart(g, out, tokens, pow2)
    dy = dy.T.contiguous()
    w8 = T._codes(g, out, inn)
    w8[empty] = 0
    dx = T._run_input_grad(dy, w8, ws, dtype)
    w = R.decode(T._as_numbers(w8, "int8"), ws, 0)
    want = dy.double() @ w
    assert want.isfinite().all()
    _close(dx, want, _carried(dy.double().abs() @ w.abs(), want, out, dtype, tokens), "dx")


@pytest.mark.parametrize("pow2", [True, False])
@pytest.mark.parametrize("code,group", [("int8", 128), ("e4m3", 0)])
@pytest.mark.parametrize("dtype,tokens,out,inn", [(BF16, 520, 8, 264), (BF16, 2000, 16, 136), (F32, 520, 72, 264), (F32, 3000, 520, 1032)])
def test_weight_grad_of_large_gradients_and_scales_far_apart(dtype, tokens, out, inn, code, group, pow2):
    g = T._gen(out + tokens)
    dy, scales, empty = _far_apart(g, tokens, out, pow2)
    x8 = T._codes(g, tokens, inn, code)
    x8[empty] = 0
    xs = scales[:, None].expand(tokens, -(-inn // group) if group else 1).contiguous()
    dw = T._run_weight_grad(dy, x8, xs, code, group, dtype)
    x = R.decode(T._as_numbers(x8, code), xs, group)
    want = dy.double().T @ x
    assert want.isfinite().all()
    _close(dw, want, _carried(dy.double().abs().T @ x.abs(), want, tokens, dtype, out), "dweight")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,out,inn", [(1, 264, 136), (5, 200, 256), (300, 520, 384), (3000, 2056, 512)])
def test_input_grad_of_scales_that_are_not_finite_or_zero(dtype, tokens, out, inn):
    """A NaN among the weight's scales makes all of dx NaN; an infinite one what its code and dy make of it; zero nothing."""
    g = T._gen(12)
    dy, _ = _rows(g, tokens, out, BF16)
    w8, ws = T._codes(g, out, inn), T._scales(g, out)
    w8[3, 0] = 0
    ws[out // 2] = 0
    some = T._run_input_grad(dy, w8, ws, dtype)
    w = R.decode(T._as_numbers(w8, "int8"), ws, 0)
    want = dy.double() @ w
    _close(some, want, T._bound(dy.double().abs() @ w.abs(), want, out, dtype, True), "dx")
    bad = ws.clone()
    bad[out - 1] = float("nan")
    assert T._run_input_grad(dy, w8, bad, dtype).isnan().all()
    bad = ws.clone()
    bad[3] = float("inf")
    dx = T._run_input_grad(dy, w8, bad, dtype)
    sign = dy[:, 3].double()[:, None] * T._as_numbers(w8, "int8")[3][None, :]
    assert dx[:, 0].isnan().all() and (dx[sign > 0] == float("inf")).all() and (dx[sign < 0] == float("-inf")).all()


# ---- scratch that was asked for with another number of tokens ----------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,more,out,inn", [(768, 8192, 2736, 1024), (598, 4096, 12904, 304), (2900, 3000, 2048, 1024), (1700, 2000, 4096, 200), (30, 40, 264, 136)])
def test_gradients_in_the_scratch_of_more_tokens_and_in_the_least(dtype, tokens, more, out, inn):
    """Parts of K that do not fit are not made, and where the numbers of the codes do not fit the call goes without: what comes out is the same
    product."""
    g = T._gen(13)
    dy, _ = _rows(g, tokens, out, BF16)
    ld = -(-inn // 16) * 16
    w8, x8 = T._codes(g, out, inn), T._codes(g, tokens, inn)
    ws, xs = T._scales(g, out), T._scales(g, tokens, -(-inn // 128))
    form = dict(x_group=128, x8_ld=ld, w8_ld=ld, dx_dtype=T.TYPE[dtype], dweight_dtype=T.TYPE[dtype])
    d, wide = A.linear8_desc(tokens, out, inn, **form), A.linear8_desc(more, out, inn, **form)
    w, x = R.decode(T._as_numbers(w8, "int8"), ws, 0), R.decode(T._as_numbers(x8, "int8"), xs, 128)
    dx, dw = torch.empty(tokens, inn, dtype=dtype, device="cuda"), torch.empty(out, inn, dtype=dtype, device="cuda")
    cases = ((A.LINEAR8_INPUT_GRAD, A.adapm_linear8_input_grad, w8, ws, dx, dy.double(), w), (A.LINEAR8_WEIGHT_GRAD, A.adapm_linear8_weight_grad, x8, xs, dw, dy.double().T, x))
    for which, call, codes, scales, result, left, right in cases:
        want, size = left @ right, left.abs() @ right.abs()
        for n in {A.adapm_linear8_scratch_bytes(d, which), A.adapm_linear8_scratch_bytes(wide, which), 9216}:
            buf = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
            try:
                call(d, dy, codes, scales, result.fill_(5), buf[:n])
            except A.AdapmError as e:
                assert e.code == -5 and n == 9216 and out * tokens > 4e6, (which, n)      # (sums too long for a form without)
                continue
            assert A.adapm_linear8_status(buf) == 0 and (buf[n:] == 0xA5).all()
            _close(result, want, T._bound(size, want, left.shape[1], dtype, True), "gradient")


# ---- the forward product ---------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,out,inn", [(1, 264, 520), (2, 264, 520), (5, 200, 256), (300, 520, 384), (3000, 2056, 512)])
def test_forward_of_scales_far_apart(dtype, tokens, out, inn):
    """Large scales of tokens beside small ones of channels, and the reverse."""
    g = T._gen(14)
    x8, w8 = T._codes(g, tokens, inn, full=True), T._codes(g, out, inn, full=True)
    for power in (96, -96):
        xs, ws = T._scales(g, tokens, pow2=False) * 2.0**power, T._scales(g, out, pow2=False) * 2.0**-power
        y = T._run_forward(x8, xs, w8, ws, dtype)
        want = R.forward(T._as_numbers(x8, "int8"), xs, T._as_numbers(w8, "int8"), ws)
        _close(y, want, want.abs() * (3.1 * 2.0**-24 + HALF[dtype] * 1.01) + 1e-37, "y")
