"""Linear layers in 8 bits on a GPU against the plain 64-bit forms (oracle/linear8_oracle.py), at the sizes, scales and layouts
where a kernel could go wrong.

Codes and scales have to be equal.  Tolerances of the products are worked out from the arithmetic: a rounding to type t is off by at most
eps(t) / 2 of the value, the forward product's sums are whole numbers, and a sum on the tensor cores is off by at most what
_tensor_sum says.
"""
import pytest

import paper_2510_09103_b200 as A
from oracle import linear8_oracle as R
from test_gpu_operators import BF16, F32, GUARD, HALF, TYPE, _close, _gen, _guards_stand, _rows, _tensor_sum

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

E4M3 = torch.float8_e4m3fn
CODE = {"int8": A.CODE_INT8, "e4m3": A.CODE_E4M3}
FORMS = [("int8", 0, False), ("int8", 0, True), ("int8", 128, False), ("int8", 128, True), ("e4m3", 0, True), ("e4m3", 128, True)]


def _bytes_at(rows, cols, ld, shift=0, fill=0x55):
    """A [rows, cols] matrix of bytes of pitch ld, `shift` bytes behind a 512-byte boundary, with guards around its rows."""
    buf = torch.full((shift + rows * ld + 64,), fill, dtype=torch.uint8, device="cuda")
    return buf[shift:shift + rows * ld].view(rows, ld)[:, :cols], buf


def _only_rows_written(m, buf, fill=0x55):
    before = m.clone()
    m.fill_(fill)
    assert (buf == fill).all(), "something was written outside the rows"
    m.copy_(before)


def _quant(x, code, group, pow2, codes_ld=None, shift=0):
    rows, cols = x.shape
    codes, buf = _bytes_at(rows, cols, codes_ld or cols, shift)
    n = -(-cols // group) if group else 1
    scales = torch.full((rows * n + 8,), GUARD, device="cuda")
    d = A.quant8_desc(rows, cols, TYPE[x.dtype], CODE[code], group, pow2, x_ld=x.stride(0) if rows > 1 else cols, codes_ld=codes_ld or cols)
    A.adapm_quant8(d, x, codes, scales)
    _only_rows_written(codes, buf)
    assert (scales[rows * n:] == GUARD).all()
    return codes, scales[:rows * n].view(rows, n)


def _as_numbers(codes, code):
    return codes.contiguous().view(E4M3 if code == "e4m3" else torch.int8).double()


def _check_quant(x, code, group, pow2, **kw):
    before = x.clone()
    codes, scales = _quant(x, code, group, pow2, **kw)
    want = R.scales_of(x, code, group, pow2)
    assert torch.equal(scales.double().nan_to_num(-1), want.nan_to_num(-1)), "scales"
    assert torch.equal(_as_numbers(codes, code), R.codes_of(x, want, code, group)), "codes"
    assert torch.equal(x.nan_to_num(3), before.nan_to_num(3))
    return codes, scales


# ---- to 8 bits and back ----------------------------------------------------------------------------------

LAYOUTS = [(1, 1, 1, 0, 0), (1, 7, 7, 0, 0), (3, 8, 8, 0, 0), (5, 127, 127, 0, 0), (5, 128, 128, 0, 0), (4, 129, 136, 0, 0), (2, 300, 304, 1, 0), (17, 64, 64, 0, 3),
           (9, 513, 513, 0, 0), (3, 1601, 1608, 0, 0), (2, 5000, 5000, 8, 0), (2, 9001, 9001, 0, 0), (1, 8200, 8200, 0, 0), (2, 33000, 33000, 0, 8), (1, 40001, 40001, 0, 0),
           (1300, 200, 200, 0, 0), (1300, 400, 408, 0, 0), (1300, 65, 65, 0, 0), (1200, 1030, 1032, 0, 0), (1200, 2048, 2048, 0, 0)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,ld,shift,code_shift", LAYOUTS)
def test_codes_and_scales_are_the_definitions(dtype, rows, cols, ld, shift, code_shift):
    x, _ = _rows(_gen(rows + cols), rows, cols, dtype, ld, shift)
    for code, group, pow2 in FORMS:
        _check_quant(x, code, group, pow2, codes_ld=-(-cols // 8) * 8 + 8 if code_shift == 0 else cols, shift=code_shift)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_codes_next_to_half_a_step(dtype):
    """Quotients on and just beside the middle of two codes, where a rounded reciprocal of the scale would decide."""
    tops = torch.tensor([127.0, 126.5, 1.0, 0.3, 3e-3, 7.7e5, 1.9375, 255.0], device="cuda").to(dtype).float()
    half = torch.arange(-127, 127, device="cuda") + 0.5
    x = torch.zeros(len(tops), 1 + 3 * len(half), dtype=dtype, device="cuda")
    x[:, 0] = tops.to(dtype)
    s = (tops.double() / 127).float()
    at = (half[None, :] * s[:, None].double()).to(dtype).float()
    up, down = torch.nextafter(at, torch.full_like(at, 9e9)), torch.nextafter(at, torch.full_like(at, -9e9))
    x[:, 1:] = torch.cat([at, up, down], 1).to(dtype)
    top = x[:, :1].float()
    x = torch.minimum(torch.maximum(x.float(), -top), top).to(dtype)
    for code, group, pow2 in FORMS:
        _check_quant(x, code, group, pow2)


def test_codes_of_every_bf16_number_below_every_maximum():
    """All mantissas of the maximum, and all numbers of its eight binades below it, of both signs."""
    m = torch.arange(128, 256, device="cuda")
    x = (m[None, None, :] / 2.0 ** torch.arange(9, device="cuda")[:, None, None]).expand(9, 128, 128).permute(1, 0, 2).reshape(128, -1).double()
    x = torch.minimum(torch.cat([m[:, None].double(), x, -x], 1), m[:, None].double()).maximum(-m[:, None].double())
    for power in (0, -7, 40, -120):
        y = (x * 2.0**power).to(BF16)
        assert torch.equal(y.double(), x * 2.0**power)
        _check_quant(y, "int8", 0, False)
        _check_quant(y.T.contiguous().T.reshape(-1, 1 + 2 * 9 * 128)[:, :129].contiguous(), "int8", 0, False)


def test_codes_on_half_a_step_of_scales_that_are_whole_numbers():
    """fp32 numbers whose quotient is half a step exactly, for scales that are no powers of two: ties go to the even code."""
    s = torch.tensor([3.0, 5.0, 7.0, 6.0, 97.0, 12345.0, 1.5, 0.375 * 2.0**-90, 3 * 2.0**60], device="cuda", dtype=torch.float64)
    x = torch.cat([127 * s[:, None], (torch.arange(-127, 127, device="cuda").double() + 0.5)[None, :] * s[:, None]], 1).float()
    assert torch.equal(x.double()[:, 5], -122.5 * s)
    codes, scales = _check_quant(x, "int8", 0, False)
    assert torch.equal(scales[:, 0].double(), s)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scales_at_the_ends_of_the_range(dtype):
    tiny = torch.finfo(dtype).smallest_normal
    tops = [0.0, tiny, tiny * 100, tiny * 127, tiny * 448, 1.0, 127.0, 127.5, 254.0, 448.0, 449.0, 896.0, 896.5, 2.0**120, torch.finfo(dtype).max]
    sub = [2.0**-133 if dtype == BF16 else 2.0**-149, 2.0**-130]
    x = torch.zeros(len(tops) + len(sub), 256, dtype=dtype, device="cuda")
    g = _gen(4)
    for i, t in enumerate(tops + sub):
        x[i] = (torch.rand(256, generator=g, device="cuda") * 2 - 1).to(dtype).float().mul(t).to(dtype)
        x[i, 7], x[i, 200] = t, -t
    for code, group, pow2 in FORMS:
        codes, scales = _check_quant(x, code, group, pow2)
        assert scales.isfinite().all() and (scales >= 2.0**-126).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", [300, 301, 3000])
def test_a_group_that_is_not_finite_comes_back_as_nan(dtype, cols):
    x = torch.randn(40, cols, generator=_gen(1), device="cuda").to(dtype)
    x[3, 5], x[7, 140], x[11, cols - 1], x[13, 0] = float("inf"), float("nan"), float("-inf"), -float("nan")
    for code, group, pow2 in FORMS:
        codes, scales = _check_quant(x, code, group, pow2)
        back = torch.empty(40, cols, device="cuda")
        A.adapm_dequant8(A.quant8_desc(40, cols, A.TYPE_F32, CODE[code], group, pow2, codes_ld=codes.stride(0)), codes, scales, back)
        lost = back.isnan()
        assert lost.any(1).nonzero()[:, 0].tolist() == [3, 7, 11, 13]
        assert lost[3].sum() == (min(128, cols) if group else cols) and (group == 0 or lost[7, 128:256].all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,ld,shift,code_shift", LAYOUTS[:14])
def test_codes_back(dtype, rows, cols, ld, shift, code_shift):
    g = _gen(cols)
    for code, group in (("int8", 0), ("int8", 128), ("e4m3", 0), ("e4m3", 128)):
        codes_ld = -(-cols // 8) * 8 + (0 if code_shift == 0 else 1)
        codes, _ = _bytes_at(rows, cols, codes_ld, code_shift)
        codes.copy_(torch.randint(0, 256, (rows, cols), generator=g, device="cuda").to(torch.uint8))
        n = -(-cols // group) if group else 1
        scales = torch.randn(rows, n, generator=g, device="cuda").exp()
        x, buf = _rows(g, rows, cols, dtype, ld, shift, 0.0)
        A.adapm_dequant8(A.quant8_desc(rows, cols, TYPE[dtype], CODE[code], group, False, x_ld=ld, codes_ld=codes_ld), codes, scales, x)
        want = R.decode(_as_numbers(codes, code), scales, group)
        _close(x, want, want.abs() * (2.0**-24 + HALF[dtype] * 1.01), "x")           # the product, and its rounding to x's type
        _guards_stand(x, buf)


def test_codes_past_32_bits_of_elements():
    """The last rows of 2^32 + 2^20 elements: their addresses need more than 32 bits."""
    rows, cols = (1 << 20) + 256, 4096
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    at = torch.tensor([0, (1 << 20) - 1, 1 << 20, rows - 1], device="cuda")
    x[at] = torch.randn(4, cols, generator=_gen(3), device="cuda").to(BF16)
    codes = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
    for group in (0, 128):
        scales = torch.empty(rows, cols // group if group else 1, device="cuda")
        d = A.quant8_desc(rows, cols, group=group, pow2=True)
        A.adapm_quant8(d, x, codes, scales)
        want = R.scales_of(x[at], "int8", group, True)
        assert torch.equal(scales[at].double(), want) and torch.equal(codes[at].double(), R.codes_of(x[at], want, "int8", group))
        assert (scales[1:4] == 1).all() and (codes[1:4] == 0).all()
        back = torch.full((rows, cols), 7.0, dtype=BF16, device="cuda")
        A.adapm_dequant8(d, codes, scales, back)
        assert torch.equal(back[at].double(), R.decode(codes[at], scales[at], group)) and (back[(1 << 20) + 1:rows - 1] == 0).all()
        del back


# ---- the products --------------------------------------------------------------------------------------------

def _codes(g, rows, cols, code="int8", pad=0, full=False):
    """Random codes, their pitch a multiple of 16.  full: every byte that is a code (int8 -128 too), else rounded normal numbers."""
    ld = -(-(cols + pad) // 16) * 16
    m, _ = _bytes_at(rows, cols, ld)
    if code == "e4m3":
        v = (torch.randn(rows, cols, generator=g, device="cuda") * 60).clamp(-448, 448).to(E4M3).view(torch.uint8)
    elif full:
        v = torch.randint(0, 256, (rows, cols), generator=g, device="cuda").to(torch.uint8)
    else:
        v = (torch.randn(rows, cols, generator=g, device="cuda") * 40).round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    m.copy_(v)
    return m


def _scales(g, *shape, pow2=True):
    s = torch.exp2(torch.randint(-9, 1, shape, generator=g, device="cuda").float())
    return s if pow2 else s * (1 + torch.rand(*shape, generator=g, device="cuda"))


def _scratch(d, which):
    return torch.full((A.adapm_linear8_scratch_bytes(d, which),), 0xFF, dtype=torch.uint8, device="cuda")


def _run_forward(x8, xs, w8, ws, dtype=BF16, pad=0, stream=None):
    tokens, inn, out = x8.shape[0], x8.shape[1], w8.shape[0]
    y, buf = _rows(None, tokens, out, dtype, out + pad, 0, 0.0) if tokens else (torch.empty(0, out, device="cuda"), None)
    d = A.linear8_desc(tokens, out, inn, y_dtype=TYPE[dtype], x8_ld=x8.stride(0), w8_ld=w8.stride(0), y_ld=out + pad)
    s = _scratch(d, A.LINEAR8_FORWARD)
    A.adapm_linear8_forward(d, x8, xs, w8, ws, y, s, stream=stream)
    assert A.adapm_linear8_status(s, stream) == 0
    _guards_stand(y, buf)
    return y


def _check_run_forward(x8, xs, w8, ws, dtype=BF16, pad=0):
    y = _run_forward(x8, xs, w8, ws, dtype, pad)
    want = R.forward(_as_numbers(x8, "int8"), xs, _as_numbers(w8, "int8"), ws)
    # the sum's rounding to fp32 (it may pass 2^24), two products, and y's type
    _close(y, want, want.abs() * (3.1 * 2.0**-24 + HALF[dtype] * 1.01) + 1e-37, "y")
    return y


SIZES = [(1, 8, 8), (1, 512, 64), (3, 264, 72), (17, 128, 128), (64, 136, 1000), (65, 1024, 16), (128, 512, 256), (130, 1600, 136), (255, 256, 2064), (256, 256, 512),
         (257, 1376, 520), (300, 2056, 384), (700, 768, 1032), (1000, 4096, 200), (2049, 640, 272)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,out,inn", SIZES)
def test_forward(dtype, tokens, out, inn):
    g = _gen(tokens * out + inn)
    pad = 8 * (tokens % 3)
    x8, w8 = _codes(g, tokens, inn, pad=pad, full=True), _codes(g, out, inn, pad=2 * pad, full=True)
    _check_run_forward(x8, _scales(g, tokens, pow2=False), w8, _scales(g, out, pow2=False), dtype, pad)


def _run_input_grad(dy, w8, ws, dtype=BF16, pad=0, stream=None):
    tokens, out, inn = dy.shape[0], w8.shape[0], w8.shape[1]
    dx, buf = _rows(None, tokens, inn, dtype, inn + pad, 0, 0.0)
    d = A.linear8_desc(tokens, out, inn, dx_dtype=TYPE[dtype], w8_ld=w8.stride(0), y_ld=dy.stride(0) if tokens > 1 else out, dx_ld=inn + pad)
    s = _scratch(d, A.LINEAR8_INPUT_GRAD)
    A.adapm_linear8_input_grad(d, dy, w8, ws, dx, s, stream=stream)
    assert A.adapm_linear8_status(s, stream) == 0
    _guards_stand(dx, buf)
    return dx


def _run_weight_grad(dy, x8, xs, code, group, dtype=BF16, pad=0, before=None, stream=None):
    tokens, out, inn = dy.shape[0], dy.shape[1], x8.shape[1]
    dw, buf = _rows(None, out, inn, dtype, inn + pad, 0, 0.0)
    if before is not None:
        dw.copy_(before)
    d = A.linear8_desc(tokens, out, inn, x_code=CODE[code], x_group=group, dweight_dtype=TYPE[dtype], accumulate=before is not None, x8_ld=x8.stride(0),
                       y_ld=dy.stride(0) if tokens > 1 else out, dweight_ld=inn + pad)
    s = _scratch(d, A.LINEAR8_WEIGHT_GRAD)
    A.adapm_linear8_weight_grad(d, dy, x8, xs, dw, s, stream=stream)
    assert A.adapm_linear8_status(s, stream) == 0
    _guards_stand(dw, buf)
    return dw


def _bound(size, want, k, dtype, exact):
    """size: the sum of the products' magnitudes.  Decoded numbers whose scale is no power of two are a product in fp32, rounded to bf16 for a gradient
    in bf16, and as three bf16 numbers, which have its 24 bits, in three times as many terms for one in fp32."""
    if dtype == F32:
        made = _tensor_sum(k, 256) if exact else _tensor_sum(3 * k, 256) + 2.0**-24
    else:
        made = _tensor_sum(k, 16384) + (0 if exact else 2.0**-8 * 1.01)
    return size * made + want.abs() * HALF[dtype] * 1.01 + 1e-37


def _check_input_grad(dy, w8, ws, dtype, exact, pad=0):
    dx = _run_input_grad(dy, w8, ws, dtype, pad)
    w = R.decode(_as_numbers(w8, "int8"), ws, 0)
    want = dy.double() @ w
    _close(dx, want, _bound(dy.double().abs() @ w.abs(), want, w8.shape[0], dtype, exact), "dx")


def _check_weight_grad(dy, x8, xs, code, group, dtype, exact, pad=0, before=None):
    dw = _run_weight_grad(dy, x8, xs, code, group, dtype, pad, before)
    x = R.decode(_as_numbers(x8, code), xs, group)
    want, size = dy.double().T @ x, dy.double().abs().T @ x.abs()
    if before is not None:
        want, size = want + before.double(), size + before.double().abs()
    _close(dw, want, _bound(size, want, dy.shape[0], dtype, exact), "dweight")


GRAD_SIZES = [(1, 8, 8), (1, 512, 64), (3, 264, 72), (63, 128, 128), (64, 136, 1000), (65, 1024, 16), (128, 512, 256), (130, 1600, 136), (257, 256, 2064), (300, 1376, 520),
              (700, 768, 1032), (1000, 2056, 200), (4100, 320, 272)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,out,inn", GRAD_SIZES)
def test_input_grad(dtype, tokens, out, inn):
    g = _gen(tokens + out * inn)
    pad = 8 * (tokens % 3)
    dy, _ = _rows(g, tokens, out, BF16, out + pad, 0)
    w8 = _codes(g, out, inn, pad=pad, full=True)
    for pow2 in (True, False):
        _check_input_grad(dy, w8, _scales(g, out, pow2=pow2), dtype, pow2, pad)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("code,group", [("int8", 0), ("int8", 128), ("e4m3", 0), ("e4m3", 128)])
@pytest.mark.parametrize("tokens,out,inn", GRAD_SIZES)
def test_weight_grad(dtype, code, group, tokens, out, inn):
    g = _gen(tokens + out * inn + group)
    pad = 8 * (tokens % 3)
    dy, _ = _rows(g, tokens, out, BF16, out + pad, 0)
    x8 = _codes(g, tokens, inn, code, pad=pad, full=code == "int8")
    n = -(-inn // group) if group else 1
    before = torch.randn(out, inn, generator=g, device="cuda").to(dtype) if tokens % 2 else None
    for pow2 in (True, False):
        _check_weight_grad(dy, x8, _scales(g, tokens, n, pow2=pow2), code, group, dtype, pow2, pad, before)


@pytest.mark.parametrize("tokens,out,inn", [(5, 512, 264), (300, 1376, 520), (1500, 2056, 1024)])
def test_gradients_in_fp32_are_as_exact_as_fp32_for_any_scales(tokens, out, inn):
    """One scale in the middle of K that is no power of two, and scales of every size: the error is that of a sum in fp32, in the norm too."""
    g = _gen(out)
    dy, _ = _rows(g, tokens, out, BF16)
    w8, x8 = _codes(g, out, inn, full=True), _codes(g, tokens, inn, full=True)
    ws, xs = _scales(g, out), _scales(g, tokens, -(-inn // 128))
    ws[out // 2], xs[tokens // 2, -1] = 0.3, 0.7
    for w_scales, x_scales in ((ws, xs), (_scales(g, out, pow2=False), _scales(g, *xs.shape, pow2=False))):
        _check_input_grad(dy, w8, w_scales, F32, False)
        _check_weight_grad(dy, x8, x_scales, "int8", 128, F32, False)
        dx = _run_input_grad(dy, w8, w_scales, F32).double()
        want = dy.double() @ R.decode(_as_numbers(w8, "int8"), w_scales, 0)
        assert (dx - want).norm() <= 5e-7 * want.norm()
        dw = _run_weight_grad(dy, x8, x_scales, "int8", 128, F32).double()
        want = dy.double().T @ R.decode(_as_numbers(x8, "int8"), x_scales, 128)
        assert (dw - want).norm() <= 5e-7 * want.norm()


@pytest.mark.parametrize("columns", [1, 3, 16])
@pytest.mark.parametrize("k", [64, 200, 1500])
def test_gradients_of_few_columns_carry_any_scale_with_16_bits(columns, k):
    """What is left in a bf16 gradient of few tokens, or few output features, is its own rounding: two roundings of a term, the second of what
    the first leaves."""
    g = _gen(columns + k)
    inn = 392
    dy, _ = _rows(g, columns, 8 * k, BF16)
    w8, ws = _codes(g, 8 * k, inn, full=True), _scales(g, 8 * k, pow2=False)
    w = R.decode(_as_numbers(w8, "int8"), ws, 0)
    want = dy.double() @ w
    _close(_run_input_grad(dy, w8, ws), want, dy.double().abs() @ w.abs() * (_tensor_sum(2 * 8 * k, 256) + 2.0**-16) + want.abs() * HALF[BF16] * 1.01, "dx")
    out = max(8, columns // 8 * 8)
    dy, _ = _rows(g, k, out, BF16)
    for code, group in (("int8", 128), ("e4m3", 0)):
        x8, xs = _codes(g, k, inn, code, full=code == "int8"), _scales(g, k, -(-inn // 128) if group else 1, pow2=False)
        x = R.decode(_as_numbers(x8, code), xs, group)
        want = dy.double().T @ x
        _close(_run_weight_grad(dy, x8, xs, code, group), want, dy.double().abs().T @ x.abs() * (_tensor_sum(2 * k, 256) + 2.0**-16) + want.abs() * HALF[BF16] * 1.01, "dweight")
