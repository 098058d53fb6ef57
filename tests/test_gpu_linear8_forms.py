"""Linear layers in 8 bits on a GPU in every form of their kernels, against the plain 64-bit forms: the sizes of linear8_forms.py, of which
test_linear8_forms_host.py says that they take the form that they stand for.  Helpers and derivations are those of test_gpu_linear8.py."""
import pytest

import paper_2510_09103_b200 as A
import linear8_forms as L
import test_gpu_linear8 as T
from oracle import linear8_oracle as R
from test_gpu_operators import BF16, F32, HALF, TYPE, _close, _gen, _rows

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

KIND = {A.TYPE_BF16: BF16, A.TYPE_F32: F32}


def _ids(s):
    return f"{s[2].replace(', ', '-').replace(' ', '-')}-{'bf16' if s[1] == A.TYPE_BF16 else 'f32'}-{s[3]}-{s[4]}-{s[5]}"


# ---- the products ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("pad", [0, 8])
@pytest.mark.parametrize("size", L.sizes(L.FORWARD), ids=_ids)
def test_forward_in_every_form(size, pad):
    """pad 8: rows of the result that start inside a sector, which leave in wide boxes."""
    _, kind, _, tokens, out, inn = size
    g = _gen(tokens + out + inn)
    x8, w8 = T._codes(g, tokens, inn, pad=2 * pad, full=True), T._codes(g, out, inn, full=True)
    T._check_run_forward(x8, T._scales(g, tokens, pow2=False), w8, T._scales(g, out, pow2=False), KIND[kind], pad)


@pytest.mark.parametrize("pow2", [True, False])
@pytest.mark.parametrize("pad", [0, 8])
@pytest.mark.parametrize("size", L.sizes(L.INPUT), ids=_ids)
def test_input_grad_in_every_form(size, pad, pow2):
    _, kind, _, tokens, out, inn = size
    g = _gen(tokens + out + inn)
    dy, _ = _rows(g, tokens, out, BF16, out + pad, 0)
    w8 = T._codes(g, out, inn, pad=2 * pad, full=True)
    T._check_input_grad(dy, w8, T._scales(g, out, pow2=pow2), KIND[kind], pow2, pad)


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("code,group,pow2,pad", [("int8", 0, False, 0), ("int8", 128, True, 8), ("e4m3", 128, False, 8), ("e4m3", 0, True, 0)])
@pytest.mark.parametrize("size", L.sizes(L.WEIGHT), ids=_ids)
def test_weight_grad_in_every_form(size, code, group, pow2, pad, add):
    _, kind, _, tokens, out, inn = size
    g = _gen(tokens + out + inn)
    dtype = KIND[kind]
    dy, _ = _rows(g, tokens, out, BF16, out + pad, 0)
    x8 = T._codes(g, tokens, inn, code, pad=2 * pad, full=code == "int8")
    xs = T._scales(g, tokens, -(-inn // group) if group else 1, pow2=pow2)
    before = (torch.randn(out, inn, generator=g, device="cuda") * 300).to(dtype) if add else None
    T._check_weight_grad(dy, x8, xs, code, group, dtype, pow2, pad, before)


# ---- added, one call behind the other ------------------------------------------------------------------------------

@pytest.mark.parametrize("size", L.sizes(L.WEIGHT), ids=_ids)
def test_gradients_that_are_added_five_times_are_there_five_times(size):
    _, kind, _, tokens, out, inn = size
    g = _gen(tokens + out + inn)
    dtype, calls = KIND[kind], 5
    dy, _ = _rows(g, tokens, out, BF16, out, 0)
    x8, xs = T._codes(g, tokens, inn), T._scales(g, tokens)
    dw = torch.full((out, inn), 100.0, dtype=dtype, device="cuda")
    d = A.linear8_desc(tokens, out, inn, dweight_dtype=TYPE[dtype], accumulate=True, x8_ld=x8.stride(0))
    scratch = T._scratch(d, A.LINEAR8_WEIGHT_GRAD)
    for _ in range(calls):
        A.adapm_linear8_weight_grad(d, dy, x8, xs, dw, scratch)
    assert A.adapm_linear8_status(scratch) == 0
    x = R.decode(T._as_numbers(x8, "int8"), xs, 0)
    one, size = dy.double().T @ x, dy.double().abs().T @ x.abs()
    want = 100 + calls * one
    # every sum's own error, and a rounding of what is there after each call, which is never above 100 + 5 |one| and what is off
    bound = calls * (size * (T._tensor_sum(tokens, 256 if dtype == F32 else 16384) + 2.0**-24) + (100 + calls * one.abs()) * HALF[dtype] * 1.02)
    _close(dw, want, bound, "dweight")


@pytest.mark.parametrize("size", L.sizes(L.WEIGHT), ids=_ids)
def test_what_nothing_is_added_to_keeps_its_value_to_the_last_bit(size):
    """The smallest numbers of the type, and the largest."""
    _, kind, _, tokens, out, inn = size
    g = _gen(tokens + out + inn)
    dtype = KIND[kind]
    info = torch.finfo(dtype)
    dy = torch.zeros(tokens, out, dtype=BF16, device="cuda")
    x8, xs = T._codes(g, tokens, inn), T._scales(g, tokens)
    before = (torch.randint(-100, 100, (out, inn), generator=g, device="cuda").double() * (info.smallest_normal * info.eps)).to(dtype)
    before[::3] = info.max
    before[1::3] = -info.smallest_normal
    assert torch.equal(T._run_weight_grad(dy, x8, xs, "int8", 0, dtype, 0, before), before)


# ---- codes of long rows ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,ld", [(2, 70000, 70000), (3, 66000, 66008), (2, 20001, 20001), (3, 30007, 30007), (2, 40001, 40001), (2, 100003, 100003), (1, 1 << 20, 1 << 20),
                                          (1300, 2049, 2049), (1200, 9000, 9000), (1190, 9001, 9001)])
def test_codes_of_long_rows(dtype, rows, cols, ld):
    """Rows of several reads, and of more columns than a CTA holds, from addresses of either kind."""
    x, _ = _rows(_gen(cols), rows, cols, dtype, ld, 0)
    x[rows // 2, cols - 1] = 50
    for code, group, pow2 in (("int8", 0, False), ("e4m3", 0, True)):
        codes, scales = T._check_quant(x, code, group, pow2, codes_ld=-(-cols // 8) * 8)
        back = torch.empty(rows, cols, dtype=dtype, device="cuda")
        A.adapm_dequant8(A.quant8_desc(rows, cols, TYPE[dtype], T.CODE[code], codes_ld=codes.stride(0) if rows > 1 else cols), codes, scales, back)
        want = R.decode(T._as_numbers(codes, code), scales, group)
        _close(back, want, want.abs() * (2.0**-24 + HALF[dtype] * 1.01), "x")
