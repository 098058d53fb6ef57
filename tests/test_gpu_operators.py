"""Dropout, the RMS norm and the head loss on a GPU against the plain 64-bit forms (oracle/operators_oracle.py), at the sizes,
masks and layouts where a kernel could go wrong.

Tolerances are worked out from the arithmetic: a rounding to type t is off by at most eps(t) / 2 of the value, a sum of n terms
in fp32 by at most 2^-24 of the terms' magnitudes per addition on the longest chain, a sum on the tensor cores as _tensor_sum
says.
"""
import math

import pytest

import paper_2510_09103_b200 as A
from oracle import operators_oracle as R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

BF16, F32 = torch.bfloat16, torch.float32
TYPE = {BF16: A.TYPE_BF16, F32: A.TYPE_F32}
HALF = {BF16: 2.0**-8, F32: 2.0**-24}          # most that a rounding is off by, relative to the value
GUARD = 777.0


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(gen, rows, cols, dtype, ld=None, shift=0, value=None, std=1.0):
    """A [rows, cols] matrix of pitch ld whose first element lies `shift` elements behind a 512-byte boundary; what lies before,
    between and behind its rows is GUARD.  Returns (matrix, whole buffer)."""
    ld = cols if ld is None else ld
    buf = torch.full((shift + rows * ld + 64,), GUARD, dtype=dtype, device="cuda")
    m = buf[shift:shift + rows * ld].view(rows, ld)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=gen, device="cuda") * std if value is None else torch.full_like(m, value))
    return m, buf


def _guards_stand(m, buf):
    before = m.clone()
    m.fill_(GUARD)
    assert (buf == GUARD).all(), "something was written outside the rows"
    m.copy_(before)


def _close(got, want, bound, what):
    got, want = got.double(), want.double()
    bad = ~((got - want).abs() <= bound)
    bad &= ~(got.isnan() & want.isnan())
    assert not bad.any(), f"{what}: {int(bad.sum())} off, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}, worst {((got - want).abs() / bound).nan_to_num().max():.3g} of its bound"


# ---- dropout -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,ld,shift,residual", [(1, 1, 1, 0, False), (1, 8, 8, 0, True), (3, 7, 9, 1, True), (5, 40, 48, 0, False),
                                                          (4, 33, 40, 0, True), (17, 64, 64, 1, False), (2, 300, 304, 8, True),
                                                          (17, 33, 33, 0, True), (16, 63, 63, 0, False), (9, 6, 6, 0, True), (11, 64, 65, 8, False), (40, 95, 95, 0, True)])
def test_dropout_against_the_generator(dtype, rows, cols, ld, shift, residual):
    g = _gen(rows * cols)
    x, xb = _rows(g, rows, cols, dtype, ld, shift)
    r, _ = _rows(g, rows, cols, dtype, cols + 8, 0) if residual else (None, None)
    y, yb = _rows(g, rows, cols, dtype, ld + 8, shift, 0.0)
    seed, offset, p = 0x1234567_89ABCDEF, (1 << 40) + 3, 0.3
    x_before = x.clone()
    A.adapm_dropout(x, r, y, TYPE[dtype], rows, cols, p, seed, offset, x_ld=ld, residual_ld=cols + 8, y_ld=ld + 8)
    keep = R.keep_mask(rows, cols, p, seed, offset).cuda()
    want = R.drop(x.double(), keep, p)
    bound = want.abs() * (2.0**-24 + 2.0**-24)              # the factor and the product
    if residual:
        want = want + r.double()
        bound = bound + want.abs() * 2.0**-24
    _close(y, want, bound + want.abs() * HALF[dtype] * 1.01, "y")
    if not residual:
        assert ((y == 0) == ~(keep & (x != 0))).all()
    assert torch.equal(x, x_before)
    _guards_stand(x, xb)
    _guards_stand(y, yb)


def test_dropout_in_place_and_its_gradient_have_one_mask():
    g = _gen(5)
    rows, cols, p = 777, 1000, 0.1
    x, _ = _rows(g, rows, cols, BF16)
    y = torch.empty_like(x)
    A.adapm_dropout(x, None, y, A.TYPE_BF16, rows, cols, p, 3, 4)
    z = x.clone()
    A.adapm_dropout(z, None, z, A.TYPE_BF16, rows, cols, p, 3, 4)
    assert torch.equal(y, z)
    r = torch.randn(rows, cols, generator=g, device="cuda").to(BF16)
    into, apart = r.clone(), torch.empty_like(r)
    A.adapm_dropout(x, into, into, A.TYPE_BF16, rows, cols, p, 3, 4)
    A.adapm_dropout(x, r, apart, A.TYPE_BF16, rows, cols, p, 3, 4)
    assert torch.equal(into, apart)
    ones = torch.ones(rows, cols, device="cuda")
    A.adapm_dropout(ones, None, ones, A.TYPE_F32, rows, cols, p, 3, 4)
    assert torch.equal(ones != 0, (y != 0) | (x == 0) & (ones != 0))
    share, n = (ones != 0).double().mean().item(), rows * cols
    q = R.least_kept(p) / 65536
    assert abs(share - (1 - q)) < 6 * math.sqrt(q * (1 - q) / n)
    other = torch.ones(rows, cols, device="cuda")
    A.adapm_dropout(other, None, other, A.TYPE_F32, rows, cols, p, 3, 5)
    both = ((other != 0) & (ones != 0)).double().mean().item()
    assert abs(both - (1 - q) ** 2) < 6 * math.sqrt(0.19 / n)


def test_dropout_ends_of_p_and_what_a_dropped_element_held():
    x = torch.tensor([[float("nan"), float("inf"), 1.0, -2.0]], device="cuda").repeat(64, 4)
    y = torch.empty_like(x)
    A.adapm_dropout(x, None, y, A.TYPE_F32, 64, 16, 0.0, 1, 1)
    assert torch.equal(y.nan_to_num(9), x.nan_to_num(9))
    A.adapm_dropout(x, None, y, A.TYPE_F32, 64, 16, 1.0, 1, 1)
    assert (y == 0).all()
    A.adapm_dropout(x, None, y, A.TYPE_F32, 64, 16, 0.5, 1, 1)
    keep = R.keep_mask(64, 16, 0.5, 1, 1).cuda()
    assert (y[~keep] == 0).all() and y[keep & x.isnan()].isnan().all() and y[keep & x.isinf()].isinf().all()


def test_dropout_step_word_moves_the_mask_of_a_captured_graph():
    x = torch.ones(64, 64, device="cuda")
    y, want = torch.empty_like(x), torch.empty_like(x)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    A.adapm_dropout(x, None, y, A.TYPE_F32, 64, 64, 0.5, 9, 100, step)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.adapm_dropout(x, None, y, A.TYPE_F32, 64, 64, 0.5, 9, 100, step)
    for k in (0, 1, 2**33):
        step.fill_(k)
        graph.replay()
        A.adapm_dropout(x, None, want, A.TYPE_F32, 64, 64, 0.5, 9, 100 + k)
        assert torch.equal(y, want)
    assert torch.equal(want.cpu() != 0, R.keep_mask(64, 64, 0.5, 9, 100 + 2**33))


def test_dropout_past_32_bits_of_elements():
    """The last elements of 2^32 + 2^20: their counters and addresses need more than 32 bits."""
    rows, cols = (1 << 20) + 256, 4096
    x = torch.ones(rows, cols, dtype=BF16, device="cuda")
    A.adapm_dropout(x, None, x, A.TYPE_BF16, rows, cols, 0.5, 2, 3)
    for row in (0, (1 << 20) - 1, 1 << 20, rows - 1):
        for g in (0, cols // 8 - 1):
            q = row * (cols // 8) + g
            w = R.philox4x32_10((q & 0xFFFFFFFF, q >> 32, 3, 0), (2, 0))
            want = [2.0 if (w[j // 2] >> (16 * (j % 2))) & 0xFFFF >= 32768 else 0.0 for j in range(8)]
            assert x[row, 8 * g:8 * g + 8].tolist() == want
    zeros = rows * cols - int((x != 0).sum())
    assert abs(zeros / (rows * cols) - 0.5) < 6 * math.sqrt(0.25 / (rows * cols))


# ---- RMS norm ------------------------------------------------------------------------------------------

NORM_SIZES = [  # rows, cols, pitch added, shift of the buffers in elements
    (1, 1, 0, 0), (1, 8, 0, 0), (3, 5, 3, 1), (2, 129, 7, 0), (5, 256, 0, 0), (1, 4096, 0, 0), (7, 1000, 8, 8), (4, 1001, 0, 0),
    (2400, 64, 0, 0), (2500, 248, 8, 0), (2400, 512, 0, 0), (2371, 1024, 0, 0), (2369, 2048, 0, 0), (2400, 333, 0, 1),
    (3, 4104, 0, 0), (2, 8192, 0, 0), (2, 8200, 0, 0), (2, 32768, 0, 0), (2, 20001, 0, 0),
    (2400, 1001, 0, 0), (2400, 255, 0, 8), (9, 2, 0, 0), (1300, 2056, 3, 0), (17, 8192, 5, 0), (9, 32761, 0, 0), (9, 32767, 0, 0), (20, 8191, 0, 0),
]


@pytest.mark.parametrize("dtype,wtype", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("rows,cols,pad,shift", NORM_SIZES)
def test_rmsnorm_forward(dtype, wtype, rows, cols, pad, shift):
    g = _gen(rows + cols)
    ld = cols + pad
    x, xb = _rows(g, rows, cols, dtype, ld, shift)
    residual, rb = _rows(g, rows, cols, dtype, ld + 8, shift, std=3.0)
    w = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(wtype)
    out = [_rows(g, rows, cols, dtype, ld, shift, 0.0) for _ in range(2)]
    (s, sb), (y, yb) = out
    rstd = torch.empty(rows, device="cuda")
    d = A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[wtype], 1e-5, x_ld=ld, residual_ld=ld + 8, sum_ld=ld, y_ld=ld)
    before = x.clone(), residual.clone()
    A.adapm_rmsnorm_forward(d, x, residual, w, s, y, None, None, rstd)
    ws, wr, wy = R.rmsnorm(x, residual, w, 1e-5)
    _close(s, ws, ws.abs() * (HALF[dtype] + 2.0**-23), "sum")
    # the sum of squares: chains of at most 8 * 8 + 15 additions, then a division, a root and a quotient
    chain = (64 + 15 + 8) * 2.0**-24
    _close(rstd, wr, wr * chain, "rstd")
    _close(y, wy, wy.abs() * (HALF[dtype] * 1.01 + chain + 2.0**-22), "y")
    assert torch.equal(x, before[0]) and torch.equal(residual, before[1])
    for m, b in ((x, xb), (residual, rb), *out):
        _guards_stand(m, b)
    # the output over the input
    if pad == 0:
        over = x.clone(memory_format=torch.contiguous_format)
        A.adapm_rmsnorm_forward(A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[wtype], 1e-5, residual_ld=ld + 8), over, residual, w, None, over, None, None, None)
        assert torch.equal(over, y)
    # the residual updated in place, no norm of it kept
    A.adapm_rmsnorm_forward(A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[wtype], 1e-5, x_ld=ld, residual_ld=ld + 8, sum_ld=ld + 8),
                            x, residual, w, residual, None, None, None, None)
    assert torch.equal(residual, s)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 128), (2, 130), (5, 1000), (4, 1001), (2400, 264), (2369, 1600), (2, 4096), (3, 9000), (2400, 1003)])
def test_rmsnorm_in_8_bits(dtype, group, rows, cols):
    g = _gen(rows * 3 + cols)
    x, _ = _rows(g, rows, cols, dtype)
    x[rows // 2] = 0                                   # a row of zeros: scale 1, values 0
    x[:, : min(cols, 128)] *= 50                       # groups of very different size
    w = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype)
    n = -(-cols // group) if group else 1
    ld = -(-cols // 8) * 8 + 8
    buf = torch.full((rows, ld), 0x5A, dtype=torch.uint8, device="cuda")
    scales, y = torch.empty(rows, n, device="cuda"), torch.empty_like(x)
    d = A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], 1e-5, q8_group=group, y8_ld=ld)
    A.adapm_rmsnorm_forward(d, x, None, w, None, y, buf, scales, None)
    assert (buf[:, cols:] == 0x5A).all()
    _, _, wy = R.rmsnorm(x, None, w, 1e-5)
    ws = R.quantize_scales(wy, group)
    fp = (64 + 15 + 8) * 2.0**-24 + 2.0**-21
    _close(scales, ws, ws * fp, "scales")
    q = buf[:, :cols].contiguous().view(torch.float8_e4m3fn).double()
    per = scales.double().repeat_interleave(group or cols, 1)[:, :cols]
    # e4m3: half a step is 2^-4 of the value, and 2^-10 below the smallest normal number
    _close(q * per, wy, wy.abs() * (2.0**-4 + 2 * fp) + per * 2.0**-10, "y8")
    assert (q.abs().amax(1) == 448).sum() == rows - 1 or group
    assert (scales[rows // 2] == 1).all() and (q[rows // 2] == 0).all()
    tight = torch.full((rows * cols + 8,), 0x5A, dtype=torch.uint8, device="cuda")       # rows one behind the other
    s3 = torch.empty_like(scales)
    A.adapm_rmsnorm_forward(A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], 1e-5, q8_group=group), x, None, w, None, None, tight, s3, None)
    q3 = tight[:rows * cols].view(rows, cols).view(torch.float8_e4m3fn).double()
    _close(s3, ws, ws * fp, "scales")
    _close(q3 * s3.double().repeat_interleave(group or cols, 1)[:, :cols], wy, wy.abs() * (2.0**-4 + 2 * fp) + per * 2.0**-10, "y8, rows one behind the other")
    assert (tight[rows * cols:] == 0x5A).all()
    alone, s2 = torch.empty_like(buf), torch.empty_like(scales)     # 8 bits only: the same numbers
    A.adapm_rmsnorm_forward(d, x, None, w, None, None, alone, s2, None)
    assert torch.equal(alone[:, :cols], buf[:, :cols]) and torch.equal(s2, scales)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(3, 7), (5, 96), (2, 1001), (17, 61), (9, 30)])
def test_rmsnorm_with_the_branchs_dropout(dtype, rows, cols):
    g = _gen(cols)
    x, _ = _rows(g, rows, cols, dtype)
    r, _ = _rows(g, rows, cols, dtype)
    w = torch.ones(cols, dtype=dtype, device="cuda")
    keep = R.keep_mask(rows, cols, 0.25, 77, 6).cuda()
    x[~keep] = float("nan")                            # what is dropped reaches nothing
    s, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    d = A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], 1e-5, drop_p=0.25, seed=77, offset=6)
    A.adapm_rmsnorm_forward(d, x, r, w, s, y, None, None, rstd)
    ws, wr, wy = R.rmsnorm(x, r, w, 1e-5, keep, 0.25)
    most = R.drop(x.double(), keep, 0.25).abs() + r.double().abs()
    _close(s, ws, ws.abs() * HALF[dtype] * 1.01 + most * 2.0**-23, "sum")
    _close(y, wy, wy.abs() * (HALF[dtype] * 1.01 + 2.0**-17) + most * 2.0**-22 * wr[:, None], "y")


def test_rmsnorm_rows_of_extreme_values():
    cols = 264
    x = torch.ones(6, cols, device="cuda")
    x[0] = 0
    x[1, 3] = float("inf")
    x[2, 5] = float("nan")
    x[3] = 1e18
    x[4] = 1e-18
    w = torch.ones(cols, device="cuda")
    y, rstd = torch.empty_like(x), torch.empty(6, device="cuda")
    q, sc = torch.empty(6, cols, dtype=torch.uint8, device="cuda"), torch.empty(6, 1, device="cuda")
    A.adapm_rmsnorm_forward(A.rmsnorm_desc(6, cols, A.TYPE_F32, A.TYPE_F32, 1e-5), x, None, w, None, y, q, sc, rstd)
    assert (y[0] == 0).all() and rstd[0].item() == pytest.approx(1e-5 ** -0.5, rel=1e-6)
    assert rstd[1] == 0 and y[1, 3].isnan() and (y[1, :3] == 0).all()
    assert y[2].isnan().all() and q[2].view(torch.float8_e4m3fn).float().isnan().all() and sc[2] == 1
    assert torch.allclose(y[3], torch.ones(cols, device="cuda"), rtol=1e-5) and torch.allclose(y[5], torch.ones(cols, device="cuda"), rtol=1e-5)
    assert torch.allclose(y[4], torch.full((cols,), 1e-18 * 1e-5 ** -0.5, device="cuda"), rtol=1e-5)


@pytest.mark.parametrize("dtype,gtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("rows,cols,pad,shift", NORM_SIZES + [(5000, 40, 0, 0), (1300, 4096, 0, 0), (5000, 41, 0, 0), (1500, 4099, 0, 0), (1200, 8195, 0, 0)])
def test_rmsnorm_backward(dtype, gtype, rows, cols, pad, shift):
    g = _gen(rows + 2 * cols)
    ld = cols + pad
    dy, dyb = _rows(g, rows, cols, dtype, ld, shift)
    dsum, _ = _rows(g, rows, cols, dtype, ld + 16, shift)
    s, _ = _rows(g, rows, cols, dtype, ld + 16, shift, std=2.0)
    w = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype)
    rstd = (s.float().square().mean(1) + 1e-5).rsqrt()
    dres, db = _rows(g, rows, cols, dtype, ld + 8, shift, 0.0)
    dw = torch.full((cols + 16,), GUARD, dtype=gtype, device="cuda")
    d = A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], 1e-5, residual_ld=ld + 8, sum_ld=ld + 16, y_ld=ld)
    scratch = torch.full((A.adapm_rmsnorm_backward_scratch_bytes(d) + 64,), 0x7F, dtype=torch.uint8, device="cuda")
    A.adapm_rmsnorm_backward(d, dy, dsum, s, rstd, w, dres, None, dw[8:], TYPE[gtype], False, scratch)
    want, _, wdw = R.rmsnorm_grad(dy, dsum, s, rstd, w)
    xh, dyw = s.double() * rstd.double()[:, None], dy.double() * w.double()
    fp = (64 + 15 + 8) * 2.0**-24
    inner = (dyw * xh).abs().mean(1, keepdim=True)
    bound = rstd.double()[:, None] * (dyw.abs() * 2.0**-21 + xh.abs() * inner * (fp + 2.0**-21)) + dsum.double().abs() * 2.0**-23
    _close(dres, want, bound + want.abs() * HALF[dtype] * 1.01, "dresidual")
    terms = (dy.double() * xh).abs().sum(0)
    wbound = terms * ((rows / 100 + 64 + 8) * 2.0**-24) + wdw.abs() * HALF[gtype] * 1.01
    _close(dw[8:8 + cols], wdw, wbound, "dweight")
    assert (dw[:8] == GUARD).all() and (dw[8 + cols:] == GUARD).all() and (scratch[-64:] == 0x7F).all()
    _guards_stand(dy, dyb)
    _guards_stand(dres, db)
    # added to what is there; without dsum; the gradient alone and the weight's alone; the same bits twice
    more = torch.randn(cols, generator=g, device="cuda").to(gtype)
    into = more.clone()
    A.adapm_rmsnorm_backward(d, dy, dsum, s, rstd, w, None, None, into, TYPE[gtype], True, scratch[:-64])
    total = more.double() + wdw
    _close(into, total, wbound + total.abs() * HALF[gtype] * 1.01 + (more.double().abs() + wdw.abs()) * 2.0**-23, "accumulated")
    apart, again = torch.empty_like(dres.contiguous()), dw[8:8 + cols].clone()
    d2 = A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], 1e-5, sum_ld=ld + 16, y_ld=ld)
    A.adapm_rmsnorm_backward(d2, dy, None, s, rstd, w, apart, None, None, A.TYPE_F32, False, None)
    _close(apart, want - dsum.double(), bound + (want - dsum.double()).abs() * HALF[dtype] * 1.01, "without dsum")
    A.adapm_rmsnorm_backward(d, dy, dsum, s, rstd, w, None, None, again, TYPE[gtype], False, scratch[:-64])
    assert torch.equal(again, dw[8:8 + cols])


@pytest.mark.parametrize("rows,cols", [(3, 7), (6, 96), (2, 9001), (19, 61), (9, 30)])
def test_rmsnorm_backward_with_dropout_and_in_place(rows, cols):
    g = _gen(cols + 1)
    dy, dsum, s = (_rows(g, rows, cols, F32)[0] for _ in range(3))
    w = torch.randn(cols, generator=g, device="cuda")
    rstd = (s.square().mean(1) + 1e-5).rsqrt()
    keep = R.keep_mask(rows, cols, 0.25, 77, 6).cuda()
    d = A.rmsnorm_desc(rows, cols, A.TYPE_F32, A.TYPE_F32, 1e-5, drop_p=0.25, seed=77, offset=6)
    dres, dx = torch.empty_like(s), torch.empty_like(s)
    A.adapm_rmsnorm_backward(d, dy, dsum, s, rstd, w, dres, dx, None, A.TYPE_F32, False, None)
    want, wdx, _ = R.rmsnorm_grad(dy, dsum, s, rstd, w, keep, 0.25)
    scale = (dy.double() * w).abs().amax() * rstd.double().amax() * 8 + dsum.abs().amax()
    _close(dres, want, scale * 2.0**-17, "dresidual")
    _close(dx, wdx, scale * 2.0**-16, "dx")
    assert (dx[~keep] == 0).all()
    a, b = dy.clone(), dsum.clone()                     # dx over dy, dresidual over dsum
    A.adapm_rmsnorm_backward(d, a, b, s, rstd, w, b, a, None, A.TYPE_F32, False, None)
    assert torch.equal(a, dx) and torch.equal(b, dres)


def test_rmsnorm_of_no_rows():
    dw = torch.ones(64, device="cuda")
    d = A.rmsnorm_desc(0, 64)
    A.adapm_rmsnorm_backward(d, None, None, None, None, None, None, None, dw, A.TYPE_F32, True, None)
    assert (dw == 1).all()
    A.adapm_rmsnorm_backward(d, None, None, None, None, None, None, None, dw, A.TYPE_F32, False, None)
    assert (dw == 0).all()


# ---- head loss -----------------------------------------------------------------------------------------

def _head_case(tokens, vocab, width, pad=0, wpad=0, shift=0, ignored=0.0, seed=0, std=0.05):
    g = _gen(1000 * seed + tokens + vocab + width)
    hidden, hb = _rows(g, tokens, width, BF16, width + pad, shift)
    weight, wb = _rows(g, vocab, width, BF16, width + wpad, shift, std=std)
    targets = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    targets[0], targets[-1] = 0, vocab - 1
    for i, at in enumerate((127, 128, 255, 256, 31, 32)):
        if tokens > i + 2 and at < vocab:
            targets[i + 1] = at
    if ignored:
        targets[torch.randperm(tokens, generator=g, device="cuda")[: int(tokens * ignored)]] = -100
        hidden[targets == -100] = float("nan")           # a padded batch
    return hidden, hb, weight, wb, targets


def _tensor_sum(n, segment):
    """What a sum of n products on the tensor cores may be off by, relative to the sum of their magnitudes.  Products of bf16
    numbers are exact; every step of 16 cuts the terms that it shifts into place and its result toward zero, each by
    at most 2^-23 of what has been summed; a segment of at most `segment` terms is one such chain, and the segments are added
    up in fp32 to nearest."""
    return (2 * (min(n, segment) / 16 + 1) + n / segment + 1) * 2.0**-23


def _logit_error(hidden, weight):
    """[tokens]: what a logit may be off by."""
    most = torch.cat([(h.double().abs() @ weight.double().abs().T).amax(1) for h in hidden.split(2048)])
    return _tensor_sum(weight.shape[1], 512) * most


def _check_forward(hidden, weight, targets, loss, lse, **kw):
    want, wlse = R.head_loss(hidden, weight, targets, **kw)
    vocab = weight.shape[0]
    ez = _logit_error(hidden, weight).nan_to_num()
    chain = (24 + vocab / 1024) * 2.0**-24 + 2.0**-21
    b = ez + chain + wlse.abs() * 2.0**-23
    _close(lse, wlse, b, "lse")
    smooth = kw.get("smooth", 0.0)
    top = hidden.double().nan_to_num().abs().sum(1) * weight.double().abs().max()
    b = b * (1 + 2 * kw.get("z_loss", 0.0) * wlse.abs()) + ez + smooth * (ez + top * (128 + vocab / 1024) * 2.0**-24) + want.abs() * 2.0**-22
    _close(loss, want, b, "loss")


def _forward(hidden, weight, targets, ld=None, wld=None, scratch=None, stream=None, **kw):
    tokens, width = hidden.shape
    d = A.head_loss_desc(tokens, weight.shape[0], width, hidden.stride(0) if ld is None else ld, weight.stride(0) if wld is None else wld, **kw)
    loss, lse = torch.full((tokens + 8,), GUARD, device="cuda"), torch.full((tokens + 8,), GUARD, device="cuda")
    n = A.adapm_head_loss_scratch_bytes(d, False)
    scratch = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda") if scratch is None else scratch
    A.adapm_head_loss_forward(d, hidden, weight, targets, loss, lse, scratch, stream=stream)
    assert A.adapm_head_loss_status(scratch, stream) == 0
    assert (scratch[n:] == 0xFF).all() and (loss[tokens:] == GUARD).all() and (lse[tokens:] == GUARD).all()
    return loss[:tokens], lse[:tokens]


HEAD_SIZES = [  # tokens, vocab, width, pad of hidden, pad of weight, shift, ignored
    (1, 1, 8, 0, 0, 0, 0), (1, 37, 8, 0, 0, 0, 0), (3, 300, 64, 8, 0, 0, 0), (128, 255, 72, 0, 8, 8, 0), (255, 257, 128, 0, 0, 0, 0.3),
    (256, 256, 256, 0, 0, 0, 0), (257, 1000, 264, 24, 8, 0, 0), (700, 5003, 520, 0, 0, 8, 0.5), (1025, 2049, 1600, 8, 0, 0, 0),
    (300, 33000, 64, 0, 0, 0, 0.9), (5000, 700, 136, 0, 0, 0, 0.01),
]


@pytest.mark.parametrize("smooth,z_loss", [(0.0, 0.0), (0.1, 1e-3)])
@pytest.mark.parametrize("tokens,vocab,width,pad,wpad,shift,ignored", HEAD_SIZES)
def test_head_loss_forward(tokens, vocab, width, pad, wpad, shift, ignored, smooth, z_loss):
    hidden, hb, weight, wb, targets = _head_case(tokens, vocab, width, pad, wpad, shift, ignored)
    loss, lse = _forward(hidden, weight, targets, width + pad, width + wpad, label_smoothing=smooth, z_loss=z_loss)
    _check_forward(hidden, weight, targets, loss, lse, smooth=smooth, z_loss=z_loss)
    _guards_stand(hidden, hb)
    _guards_stand(weight, wb)


def _backward(hidden, weight, targets, lse, dloss=None, scale=1.0, dht=BF16, dwt=BF16, want_dh=True, want_dw=True, into=None, ld=None, wld=None,
              shift=0, **kw):
    tokens, width = hidden.shape
    vocab = weight.shape[0]
    ld, wld = hidden.stride(0) if ld is None else ld, weight.stride(0) if wld is None else wld
    d = A.head_loss_desc(tokens, vocab, width, ld, wld, dhidden_dtype=TYPE[dht], dweight_dtype=TYPE[dwt], accumulate=into is not None, **kw)
    n = A.adapm_head_loss_scratch_bytes(d, True)
    scratch = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")     # NaN wherever it is read before it is written
    dh, dhb = _rows(None, tokens, width, dht, ld, shift, 5.0) if want_dh else (None, None)
    dw, dwb = _rows(None, vocab, width, dwt, wld, shift, 5.0) if want_dw else (None, None)
    if into is not None:
        dw.copy_(into)
    A.adapm_head_loss_backward(d, hidden, weight, targets, lse, dloss, scale, dh, dw, scratch)
    assert A.adapm_head_loss_status(scratch) == 0
    assert (scratch[n:] == 0xFF).all()
    for m, b in ((dh, dhb), (dw, dwb)):
        if m is not None:
            _guards_stand(m, b)
    return dh, dw


def _check_backward(hidden, weight, targets, lse, dh, dw, dloss=None, scale=1.0, into=None, ignore=-100, smooth=0.0, z_loss=0.0):
    kw = dict(ignore=ignore, smooth=smooth, z_loss=z_loss)
    at, g = R.head_logit_grad(hidden, weight, targets, lse, dloss, scale, **kw)
    h, w = hidden[at].double(), weight.double()
    dl = torch.ones(len(at), dtype=torch.float64, device="cuda") if dloss is None else dloss[at].double().abs()
    ez = _logit_error(hidden[at], weight)[:, None] if len(at) else torch.zeros(0, 1, dtype=torch.float64, device="cuda")
    l = lse[at].double()[:, None]
    p = torch.exp(h @ w.T - l) * (1 + 2 * z_loss * l).abs()
    hit = torch.zeros_like(g)
    hit[torch.arange(len(at), device="cuda"), targets[at]] = 1
    made = scale * dl[:, None] * (p * (2 * ez + 2.0**-19 + l.abs() * 2.0**-22) + (smooth / weight.shape[0] + hit) * 2.0**-22)
    for out, kind in ((dh, "dhidden"), (dw, "dweight")):
        if out is None:
            continue
        bound = made + g.abs() * (2.0**-8 if out.dtype == BF16 else 2.0**-22)
        segment = 4096 if out.dtype == BF16 else 256
        if kind == "dhidden":
            want = torch.zeros(hidden.shape, dtype=torch.float64, device="cuda")
            b = torch.zeros_like(want)
            want[at] = g @ w
            b[at] = (bound + g.abs() * _tensor_sum(weight.shape[0], segment)) @ w.abs()
            if dh is not None and len(at) < len(targets):
                rest = torch.ones(len(targets), dtype=torch.bool, device="cuda")
                rest[at] = False
                assert (dh[rest] == 0).all()
        else:
            want = g.T @ h
            b = (bound + g.abs() * _tensor_sum(len(at), segment)).T @ h.abs()
            if into is not None:
                want = want + into.double()
                b = b + into.double().abs() * 2.0**-23
        _close(out, want, b + want.abs() * (HALF[out.dtype] * 1.01 + 2.0**-22) + 1e-30, kind)


@pytest.mark.parametrize("dht,dwt", [(BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)])
@pytest.mark.parametrize("tokens,vocab,width,pad,wpad,shift,ignored", HEAD_SIZES)
def test_head_loss_backward(tokens, vocab, width, pad, wpad, shift, ignored, dht, dwt):
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width, pad, wpad, shift, ignored)
    kw = dict(label_smoothing=0.1, z_loss=1e-3) if width % 16 == 0 else {}
    rw = dict(smooth=0.1, z_loss=1e-3) if kw else {}
    lse = R.head_loss(hidden, weight, targets, **rw)[1].float()
    g = _gen(9)
    dloss = torch.randn(tokens, generator=g, device="cuda") if tokens % 2 else None
    if dloss is not None and ignored:
        dloss[targets == -100] = float("nan")
    dh, dw = _backward(hidden, weight, targets, lse, dloss, 0.37, dht, dwt, ld=width + pad, wld=width + wpad, shift=shift, **kw)
    _check_backward(hidden, weight, targets, lse, dh, dw, dloss, 0.37, **rw)


@pytest.mark.parametrize("dht,dwt", [(BF16, BF16), (F32, F32)])
def test_head_loss_backward_over_several_pieces_of_the_vocabulary(dht, dwt):
    """32768 tokens: pieces of 2048 columns, three of them, the last one short; the sum of dhidden goes through memory."""
    tokens, vocab, width = 32768, 4400, 72
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width, ignored=0.2, std=0.3)
    lse = R.head_loss(hidden, weight, targets)[1].float()
    into = torch.randn(vocab, width, device="cuda").to(dwt)
    dh, dw = _backward(hidden, weight, targets, lse, None, 1.0 / tokens, dht, dwt, into=into)
    _check_backward(hidden, weight, targets, lse, dh, dw, None, 1.0 / tokens, into=into)


@pytest.mark.parametrize("dht,dwt", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("tokens,vocab,width,ignored", [(2000, 40000, 72, 0.1), (5000, 700, 136, 0.3), (5000, 700, 136, 0.99), (40, 9000, 264, 0.0)])
def test_head_loss_backward_where_the_long_side_of_a_product_is_cut(tokens, vocab, width, ignored, dht, dwt):
    """Few tiles with a long K: dhidden over two pieces in several parts each, dweight in parts (with fewer tokens than they were
    planned for, too), and both added to what is there."""
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width, ignored=ignored, std=0.3)
    lse = R.head_loss(hidden, weight, targets)[1].float()
    into = torch.randn(vocab, width, device="cuda").to(dwt)
    dh, dw = _backward(hidden, weight, targets, lse, None, 0.25, dht, dwt, into=into)
    _check_backward(hidden, weight, targets, lse, dh, dw, None, 0.25, into=into)
    assert torch.equal(_backward(hidden, weight, targets, lse, None, 0.25, dht, dwt, want_dw=False)[0], dh)
    assert torch.equal(_backward(hidden, weight, targets, lse, None, 0.25, dht, dwt, want_dh=False, into=into)[1], dw)


def test_head_loss_one_gradient_alone_and_the_same_bits_twice():
    hidden, _, weight, _, targets = _head_case(600, 3001, 96, ignored=0.2)
    lse = R.head_loss(hidden, weight, targets)[1].float()
    dh, dw = _backward(hidden, weight, targets, lse)
    assert torch.equal(_backward(hidden, weight, targets, lse, want_dw=False)[0], dh)
    assert torch.equal(_backward(hidden, weight, targets, lse, want_dh=False)[1], dw)
    noise, side = torch.zeros(1 << 24, device="cuda"), torch.cuda.Stream()
    for _ in range(10):
        with torch.cuda.stream(side):
            noise.add_(1)
        a, b = _backward(hidden, weight, targets, lse)
        assert torch.equal(a, dh) and torch.equal(b, dw)


@pytest.mark.parametrize("where", ["ignored", "out of range"])
def test_head_loss_without_any_target(where):
    hidden, _, weight, _, targets = _head_case(300, 1000, 64)
    targets.fill_(-100 if where == "ignored" else 1000)
    hidden.fill_(float("nan"))
    loss, lse = _forward(hidden, weight, targets)
    assert (loss == 0).all() and (lse == 0).all() if where == "ignored" else loss.isnan().all() and lse.isnan().all()
    dh, dw = _backward(hidden, weight, targets, lse)
    assert (dh == 0).all() and (dw == 0).all()
    into = torch.randn(1000, 64, device="cuda").to(BF16)
    assert torch.equal(_backward(hidden, weight, targets, lse, into=into)[1], into)


def test_head_loss_targets_out_of_range_and_an_index_inside_the_vocabulary_that_is_ignored():
    hidden, _, weight, _, targets = _head_case(300, 1000, 64)
    targets[5], targets[6], targets[7] = 1000, -1, 2**40
    loss, lse = _forward(hidden, weight, targets, ignore_index=0)
    assert loss[5:8].isnan().all() and loss[0] == 0 and targets[0] == 0
    _check_forward(hidden, weight, targets, loss, lse, ignore=0)
    dh, dw = _backward(hidden, weight, targets, lse, ignore_index=0)
    _check_backward(hidden, weight, targets, lse, dh, dw, ignore=0)


def test_head_loss_of_no_tokens():
    weight = torch.ones(50, 64, dtype=BF16, device="cuda")
    d = A.head_loss_desc(0, 50, 64)
    A.adapm_head_loss_forward(d, None, weight, None, None, None, None)
    dw = torch.ones(50, 64, dtype=BF16, device="cuda")
    A.adapm_head_loss_backward(A.head_loss_desc(0, 50, 64, accumulate=1), None, weight, None, None, None, 1.0, None, dw, None)
    assert (dw == 1).all()
    A.adapm_head_loss_backward(d, None, weight, None, None, None, 1.0, None, dw, None)
    assert (dw == 0).all()


def test_head_loss_of_large_and_infinite_logits():
    hidden, _, weight, _, targets = _head_case(64, 500, 64, std=40.0)
    hidden *= 8
    loss, lse = _forward(hidden, weight, targets)
    want, wlse = R.head_loss(hidden, weight, targets)
    assert lse.max() > 3000
    _check_forward(hidden, weight, targets, loss, lse)
    dh, dw = _backward(hidden, weight, targets, lse)
    assert dh.isfinite().all() and dw.isfinite().all()
    weight[17] = float("-inf")
    weight[18, 0] = float("nan")
    hidden[:, 0] = hidden[:, 0].abs()
    hidden[3:] = 0
    hidden[3:, 1] = 0
    loss, _ = _forward(hidden, weight, targets)
    assert loss.isnan().all()                      # a NaN in the weight reaches every logit's sum, as in the plain form


def test_head_loss_on_another_stream_and_in_a_graph():
    hidden, _, weight, _, targets = _head_case(700, 5003, 520, ignored=0.3)
    loss, lse = _forward(hidden, weight, targets)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other, _ = _forward(hidden, weight, targets)
    side.synchronize()
    assert torch.equal(other, loss)
    given, _ = _forward(hidden, weight, targets, stream=side)
    side.synchronize()
    assert torch.equal(given, loss)
    tokens, width = hidden.shape
    d = A.head_loss_desc(tokens, 5003, width)
    sf, sb = (torch.empty(A.adapm_head_loss_scratch_bytes(d, b), dtype=torch.uint8, device="cuda") for b in (False, True))
    out = [torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty_like(hidden), torch.empty_like(weight)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.adapm_head_loss_forward(d, hidden, weight, targets, out[0], out[1], sf)
        A.adapm_head_loss_backward(d, hidden, weight, targets, out[1], None, 0.5, out[2], out[3], sb)
    for seed in (1, 2):
        h, _, w, _, t = _head_case(700, 5003, 520, ignored=0.1 * seed, seed=seed)      # another number of targets
        hidden.copy_(h); weight.copy_(w); targets.copy_(t)
        graph.replay()
        loss, lse = _forward(hidden, weight, targets)
        assert torch.equal(out[0], loss) and torch.equal(out[1], lse)
        dh, dw = _backward(hidden, weight, targets, lse, None, 0.5)
        assert torch.equal(out[2], dh) and torch.equal(out[3], dw)


def test_head_loss_twice_at_once():
    """Two calls on two streams, each with a scratch of its own, again and again."""
    cases = [_head_case(700, 5003, 520, ignored=0.3), _head_case(300, 9001, 264, seed=1)]
    want = [(_forward(h, w, t)[0], _backward(h, w, t, R.head_loss(h, w, t)[1].float())) for h, _, w, _, t in cases]
    lses = [R.head_loss(h, w, t)[1].float() for h, _, w, _, t in cases]
    streams, out = [torch.cuda.Stream() for _ in cases], [[], []]
    held = []
    for i, (h, _, w, _, t) in enumerate(cases):
        d = A.head_loss_desc(h.shape[0], w.shape[0], h.shape[1])
        held.append((d, torch.empty(A.adapm_head_loss_scratch_bytes(d, False), dtype=torch.uint8, device="cuda"),
                     torch.empty(A.adapm_head_loss_scratch_bytes(d, True), dtype=torch.uint8, device="cuda")))
        out[i] = [[torch.empty(h.shape[0], device="cuda"), torch.empty(h.shape[0], device="cuda"), torch.empty_like(h.contiguous()), torch.empty_like(w.contiguous())] for _ in range(6)]
    torch.cuda.synchronize()
    for k in range(6):
        for i, (h, _, w, _, t) in enumerate(cases):
            d, sf, sb = held[i]
            o = out[i][k]
            A.adapm_head_loss_forward(d, h, w, t, o[0], o[1], sf, stream=streams[i])
            A.adapm_head_loss_backward(d, h, w, t, lses[i], None, 1.0, o[2], o[3], sb, stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for o in out[i]:
            assert torch.equal(o[0], want[i][0]) and torch.equal(o[2], want[i][1][0]) and torch.equal(o[3], want[i][1][1])


def test_head_loss_past_32_bits_of_weight_elements():
    """2.2e9 elements of weight: the last rows' addresses need more than 32 bits."""
    tokens, vocab, width = 5, 540000, 4096
    g = _gen(8)
    weight = torch.empty(vocab, width, dtype=BF16, device="cuda")
    for part in weight.split(20000):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * 0.02)
    hidden = torch.randn(tokens, width, generator=g, device="cuda").to(BF16)
    targets = torch.tensor([vocab - 1, 0, 524288, vocab - 2, 300000], device="cuda")
    loss, lse = _forward(hidden, weight, targets)
    z = torch.cat([hidden.double() @ part.double().T for part in weight.split(20000)], 1)
    want = torch.logsumexp(z, 1)
    err = _tensor_sum(width, 512) * 4096 * 0.02 * 5 * 5 + 600 * 2.0**-24 + 2.0**-20      # (no product above 25 times its mean size)
    assert ((lse.double() - want).abs() < err).all()
    assert ((loss.double() - want + z.gather(1, targets[:, None])[:, 0]).abs() < 2 * err).all()
    d = A.head_loss_desc(tokens, vocab, width)
    scratch = torch.empty(A.adapm_head_loss_scratch_bytes(d, True), dtype=torch.uint8, device="cuda")
    dw, dh = torch.full_like(weight, 7.0), torch.empty_like(hidden)
    A.adapm_head_loss_backward(d, hidden, weight, targets, lse, None, 1.0, dh, dw, scratch)
    grad = torch.exp(z - lse.double()[:, None])
    grad[torch.arange(tokens, device="cuda"), targets] -= 1
    for rows in (slice(0, 300), slice(524200, 524400), slice(vocab - 300, vocab)):
        ref = grad[:, rows].T @ hidden.double()
        assert (dw[rows].double() - ref).norm() < 4e-3 * ref.norm()          # two roundings of 2^-8 at most, 1.7e-3 in the norm each
    ref = sum(grad[:, i:i + 20000] @ weight[i:i + 20000].double() for i in range(0, vocab, 20000))
    assert (dh.double() - ref).norm() < 4e-3 * ref.norm()
    assert dw.isfinite().all() and (dw[::1013] != 7.0).any(1).all()


def test_rmsnorm_past_32_bits_of_elements():
    """The last rows of 2.3e9 elements are what the same rows give by themselves."""
    rows, cols = 70000, 32768
    x = torch.empty(rows, cols, dtype=BF16, device="cuda")
    x.normal_(generator=_gen(9))
    w = torch.ones(cols, dtype=BF16, device="cuda")
    rstd, y = torch.empty(rows, device="cuda"), torch.empty_like(x)
    A.adapm_rmsnorm_forward(A.rmsnorm_desc(rows, cols), x, None, w, None, y, None, None, rstd)
    tail = x[-8:].clone()
    alone, r = torch.empty_like(tail), torch.empty(8, device="cuda")
    A.adapm_rmsnorm_forward(A.rmsnorm_desc(8, cols), tail, None, w, None, alone, None, None, r)
    assert torch.equal(y[-8:], alone) and torch.equal(rstd[-8:], r) and y[65536 + 1].isfinite().all()
    A.adapm_rmsnorm_backward(A.rmsnorm_desc(rows, cols), y, None, x, rstd, w, y, None, None, A.TYPE_F32, False, None)
    A.adapm_rmsnorm_backward(A.rmsnorm_desc(8, cols), alone, None, tail, r, w, alone, None, None, A.TYPE_F32, False, None)
    assert torch.equal(y[-8:], alone)


FIRST_CALL_IN_A_CAPTURE = """
import torch, paper_2510_09103_b200 as A
b = torch.bfloat16
x, w, y = torch.randn(64, 512, device="cuda").to(b), torch.randn(300, 512, device="cuda").to(b), torch.zeros(64, 512, dtype=b, device="cuda")
t, out = torch.randint(0, 300, (64,), device="cuda"), torch.zeros(6, 64, device="cuda")
ones = torch.ones(512, dtype=b, device="cuda")
nd, hd = A.rmsnorm_desc(64, 512, drop_p=0.1), A.head_loss_desc(64, 300, 512)
s = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (A.adapm_head_loss_scratch_bytes(hd, False), A.adapm_head_loss_scratch_bytes(hd, True), A.adapm_rmsnorm_backward_scratch_bytes(nd))]
g = [torch.zeros_like(v) for v in (x, w, x, ones, x, y)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
def calls(g, y, out):
    A.adapm_dropout(x, None, g[5], A.TYPE_BF16, 64, 512, 0.1, 1, 1)
    A.adapm_rmsnorm_forward(nd, g[5], x, ones, g[4], y, None, None, out[0])
    A.adapm_head_loss_forward(hd, y, w, t, out[1], out[2], s[0])
    A.adapm_head_loss_backward(hd, y, w, t, out[2], None, 1.0, g[0], g[1], s[1])
    A.adapm_rmsnorm_backward(nd, g[0], None, g[4], out[0], ones, g[2], None, g[3], A.TYPE_BF16, False, s[2])
with torch.cuda.graph(graph):
    calls(g, y, out)
graph.replay()
torch.cuda.synchronize()
again, y2, out2 = [torch.zeros_like(v) for v in g], torch.zeros_like(y), torch.zeros_like(out)
calls(again, y2, out2)
torch.cuda.synchronize()
assert torch.equal(out, out2) and torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(g, again)) and out[1].isfinite().all() and out[1].any()
print("same")
"""


def test_the_first_call_of_a_process_may_be_a_captured_one():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL_IN_A_CAPTURE], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


def test_operators_refuse_memory_that_is_not_the_devices():
    host = torch.zeros(64, 64, dtype=BF16)
    dev = torch.zeros(64, 64, dtype=BF16, device="cuda")
    for call in (lambda: A.adapm_dropout(host, None, dev, A.TYPE_BF16, 64, 64, 0.1, 1, 1),
                 lambda: A.adapm_rmsnorm_forward(A.rmsnorm_desc(64, 64), dev, None, host, None, dev, None, None, None),
                 lambda: A.adapm_head_loss_forward(A.head_loss_desc(64, 64, 64), dev, dev, torch.zeros(64, dtype=torch.int64),
                                                   torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda"),
                                                   torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(A.AdapmError) as e:
            call()
        assert e.value.code == -1 and "current device" in str(e.value)


# ---- together ------------------------------------------------------------------------------------------

def test_the_tail_of_a_training_step():
    """Dropout of a branch, residual, norm, head loss and back, the gradients of the norm's and the head's weight written where
    adapm_step reads them, and the step itself: as a training program runs them, against the plain forms."""
    tokens, width, vocab, p = 512, 128, 1000, 0.1
    blocks = [A.adapm_block(0, vocab, width, A.MOM_NONE, 0, A.V_BLOCKMEAN, 1, 0.75, 0.0),
              A.adapm_block(vocab * width, 1, width, A.MOM_FULL, 0, A.V_BLOCKMEAN, 0, 1.0, 0.0)]
    ctx = A.adapm_create(blocks, A.hparams(lr=1e-2, grad_dtype=A.GRAD_BF16))
    n = vocab * width + width
    g = _gen(3)
    params = torch.cat([torch.randn(vocab * width, generator=g, device="cuda") * 0.02, torch.ones(width, device="cuda")])
    shadow, grads = params.to(BF16), torch.zeros(n, dtype=BF16, device="cuda")
    state, work = (torch.zeros(max(64, b // 4), device="cuda") for b in (ctx.adapm_state_bytes(), ctx.adapm_workspace_bytes()))
    ctx.adapm_set_workspace(work)
    ctx.adapm_set_shadow_params(shadow)
    ctx.adapm_state_init(state)
    branch, stream = (torch.randn(tokens, width, generator=g, device="cuda").to(BF16) for _ in range(2))
    targets = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    targets[::7] = -100
    head, norm_w = shadow[:vocab * width].view(vocab, width), shadow[vocab * width:]
    dhead, dnorm = grads[:vocab * width].view(vocab, width), grads[vocab * width:]
    s, y, dy, dres, dx = (torch.empty_like(stream) for _ in range(5))
    rstd, loss, lse = (torch.empty(tokens, device="cuda") for _ in range(3))
    hd = A.head_loss_desc(tokens, vocab, width)
    sf, sb = (torch.empty(A.adapm_head_loss_scratch_bytes(hd, b), dtype=torch.uint8, device="cuda") for b in (False, True))
    valid = int((targets != -100).sum())
    for t in range(1, 5):
        nd = A.rmsnorm_desc(tokens, width, drop_p=p, seed=5, offset=t)
        sn = torch.empty(A.adapm_rmsnorm_backward_scratch_bytes(nd), dtype=torch.uint8, device="cuda")
        A.adapm_rmsnorm_forward(nd, branch, stream, norm_w, s, y, None, None, rstd)
        A.adapm_head_loss_forward(hd, y, head, targets, loss, lse, sf)
        A.adapm_head_loss_backward(hd, y, head, targets, lse, None, 1.0 / valid, dy, dhead, sb)
        A.adapm_rmsnorm_backward(nd, dy, None, s, rstd, norm_w, dres, dx, dnorm, A.TYPE_BF16, False, sn)
        if t in (1, 4):
            keep = R.keep_mask(tokens, width, p, 5, t).cuda()
            _check_forward(y, head, targets, loss, lse)
            _check_backward(y, head, targets, lse, dy, dhead, None, 1.0 / valid)
            want = R.rmsnorm_grad(dy, None, s, rstd, norm_w, keep, p)
            for got, ref in zip((dres, dx, dnorm), want):
                _close(got, ref, ref.abs() * 2.0**-8 * 1.01 + ref.abs().amax() * 2.0**-14, "norm gradient")
        before = params.clone()
        ctx.adapm_step(params, grads, state, t)
        assert not torch.equal(before, params) and torch.equal(shadow, params.to(BF16))
        assert loss.isfinite().all()
    assert ctx.adapm_get_status() == 0 and A.adapm_head_loss_status(sb) == 0
    ctx.close()


def test_the_head_losss_gradient_is_the_difference_of_two_losses():
    """The forward kernel on either side along random directions.  The gradient kernel's dot product with the direction has to be
    the difference quotient up to the third derivative (|d|^3 / 6 of a logit's change d, whose third derivative of
    log-sum-exp is at most 1), and to the losses' own errors over the step."""
    tokens, vocab, width = 256, 700, 64
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width, std=0.1)
    loss, lse = _forward(hidden, weight, targets)
    dh, dw = _backward(hidden, weight, targets, lse, None, 1.0, F32, F32)
    g = _gen(4)
    for what in ("hidden", "weight"):
        base = hidden if what == "hidden" else weight
        size = 2.0**-5 if what == "hidden" else 2.0**-8
        move = torch.randn(base.shape, generator=g, device="cuda") * size
        up, down = (base + move).to(BF16), (base - move).to(BF16)
        moved = (up.double() - down.double()) / 2
        lu, ld_ = ((_forward(up, weight, targets) if what == "hidden" else _forward(hidden, up, targets))[0].double(),
                   (_forward(down, weight, targets) if what == "hidden" else _forward(hidden, down, targets))[0].double())
        middle = (up.double() + down.double()) / 2             # rounding moves the middle: the gradient there, from the formula
        m_h, m_w = (middle, weight.double()) if what == "hidden" else (hidden.double(), middle)
        at_middle = R.head_loss_grad(m_h, m_w, targets, R.head_loss(m_h, m_w, targets)[1])[0 if what == "hidden" else 1]
        d = (moved @ weight.double().T if what == "hidden" else hidden.double() @ moved.T).abs().amax(1)
        bound = (d**3 / 6).sum() + 2 * _logit_error(hidden, weight).sum() + tokens * 2.0**-19
        assert abs((lu - ld_).sum() / 2 - (at_middle * moved).sum()) <= bound
        # and the kernel's gradient at the point itself, as far as the middle is from it
        kernel = dh if what == "hidden" else dw
        drift = (at_middle - R.head_loss_grad(hidden, weight, targets, lse)[0 if what == "hidden" else 1]).abs()
        assert ((kernel.double() - at_middle).abs() <= drift + 2.0**-12 * (1 + at_middle.abs().amax())).all()
