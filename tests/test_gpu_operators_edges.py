"""Dropout, the RMS norm and the head loss on a GPU at calls that the documentation allows and that lie between the cases of
test_gpu_operators.py, whose helpers and derivations these use."""
import pytest

import paper_2510_09103_b200 as A
import test_gpu_operators as T
from oracle import operators_oracle as R
from test_gpu_operators import BF16, F32, GUARD, HALF, TYPE, _backward, _check_backward, _check_forward, _close, _forward, _gen, _head_case, _rows

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---- head loss: dhidden over pieces of different lengths -------------------------------------------------

@pytest.mark.parametrize("tokens,vocab,width,dht,dwt", [(100, 262208, 256, BF16, BF16), (100, 265792, 64, BF16, BF16), (70, 268864, 128, BF16, BF16)])
def test_head_loss_dhidden_where_the_last_piece_is_a_little_shorter(tokens, vocab, width, dht, dwt):
    """Two pieces whose K is cut into dozens of parts, the last one a few stages shorter; the targets lie where its last parts do."""
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width)
    targets[1::2] = vocab - 1 - 16 * torch.arange(len(targets[1::2]), device="cuda")
    lse = R.head_loss(hidden, weight, targets)[1].float()
    dh, dw = _backward(hidden, weight, targets, lse, None, 0.5, dht, dwt)
    _check_backward(hidden, weight, targets, lse, dh, dw, None, 0.5)


# ---- head loss: few tokens with a target among many -------------------------------------------------------

@pytest.mark.parametrize("tokens,valid", [(64, 64), (64, 1), (65, 1), (100, 10), (100, 64), (257, 1), (300, 10), (700, 64), (5000, 1), (5000, 64)])
@pytest.mark.parametrize("dht,dwt", [(BF16, BF16), (BF16, F32), (F32, BF16)])
def test_head_loss_gradient_of_few_tokens_with_a_target(tokens, valid, dht, dwt):
    """Up to 64 tokens with a target, however many others there are, the logits' gradient is carried with 16 bits into a bf16
    gradient: what is left is the gradient's own rounding.  Every token's weight is chosen so that its target's element of the
    logits' gradient lies just below the middle of two neighbouring bf16 numbers, where rounding it once costs the most."""
    vocab, width = 1000, 256
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width)
    targets = torch.randperm(vocab, generator=_gen(5), device="cuda")[:valid].repeat(-(-tokens // valid))[:tokens]
    kept = torch.randperm(tokens, generator=_gen(6), device="cuda")[:valid]
    ignored = torch.ones(tokens, dtype=torch.bool, device="cuda")
    ignored[kept] = False
    targets[ignored] = -100
    lse = R.head_loss(hidden, weight, targets)[1].float()
    at, g = R.head_logit_grad(hidden, weight, targets, lse)
    dloss = torch.zeros(tokens, device="cuda")
    dloss[at] = ((1 + 2.0**-8) * (1 - 2.0**-13) / g[torch.arange(valid, device="cuda"), targets[at]].abs()).float()
    dh, dw = _backward(hidden, weight, targets, lse, dloss, 1.0, dht, dwt)
    at, g = R.head_logit_grad(hidden, weight, targets, lse, dloss)
    h, w = hidden[at].double(), weight.double()
    l = lse[at].double()[:, None]
    hit = torch.zeros_like(g)
    hit[torch.arange(valid, device="cuda"), targets[at]] = 1
    ez = T._logit_error(hidden[at], weight)[:, None]
    made = dloss[at].double()[:, None] * (torch.exp(h @ w.T - l) * (2 * ez + 2.0**-19 + l.abs() * 2.0**-22) + hit * 2.0**-22)
    # two roundings to bf16, the second of what the first leaves (at most 2^-8 of it): 2^-16
    for out, want, size in ((dh, g @ w, lambda b: b @ w.abs()), (dw, g.T @ h, lambda b: b.T @ h.abs())):
        n = vocab if out is dh else valid
        bound = size(made + g.abs() * (2.0**-16 + T._tensor_sum(2 * n, 4096)))
        got = dh[at] if out is dh else dw
        _close(got, want, bound + want.abs() * HALF[out.dtype] * 1.01 + 1e-30, "dhidden" if out is dh else "dweight")
    assert (dh[ignored] == 0).all()


@pytest.mark.parametrize("dht,dwt", [(BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("tokens,vocab,width,ignored", [(32768, 4400, 72, 0.999), (2000, 40000, 72, 0.98), (100, 262208, 256, 0.5), (130, 262208, 64, 0.6), (8192, 20000, 520, 0.995)])
def test_head_loss_gradient_of_few_targets_over_pieces_and_parts(tokens, vocab, width, ignored, dht, dwt):
    """Two planes of few tokens as rows of one tile, summed over several pieces of the vocabulary, cut or not."""
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width, ignored=ignored, std=0.3)
    valid = int((targets != -100).sum())
    assert valid <= 64
    lse = R.head_loss(hidden, weight, targets)[1].float()
    into = torch.randn(vocab, width, device="cuda").to(dwt)
    dh, dw = _backward(hidden, weight, targets, lse, None, 0.25, dht, dwt, into=into)
    _check_backward(hidden, weight, targets, lse, dh, dw, None, 0.25, into=into)
    # the tokens by themselves: the same sums, in another order at most
    at = (targets != -100).nonzero()[:, 0]
    alone, _ = _backward(hidden[at].contiguous(), weight, targets[at].contiguous(), lse[at].contiguous(), None, 0.25, dht, dwt, want_dw=False)
    _close(dh[at], alone.double(), alone.double().abs() * 2 * HALF[dht] + alone.double().abs().amax(1, keepdim=True) * 2.0**-12, "alone")


@pytest.mark.parametrize("dht", [BF16, F32])
def test_head_loss_gradient_captured_with_many_targets_and_replayed_with_few(dht):
    """How the planes lie and what is summed follows from the targets of the replay, not from those of the capture."""
    tokens, vocab, width = 700, 5003, 520
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width)
    hidden, weight = hidden.contiguous(), weight.contiguous()
    lse = R.head_loss(hidden, weight, targets)[1].float()
    d = A.head_loss_desc(tokens, vocab, width, dhidden_dtype=TYPE[dht])
    scratch = torch.empty(A.adapm_head_loss_scratch_bytes(d, True), dtype=torch.uint8, device="cuda")
    dh, dw = torch.empty(tokens, width, dtype=dht, device="cuda"), torch.empty_like(weight)
    A.adapm_head_loss_backward(d, hidden, weight, targets, lse, None, 0.5, dh, dw, scratch)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.adapm_head_loss_backward(d, hidden, weight, targets, lse, None, 0.5, dh, dw, scratch)
    whole = targets.clone()
    for n in (700, 1, 64, 65, 0, 256, 257, 33):
        kept = torch.randperm(tokens, generator=_gen(n), device="cuda")[:n]
        targets.fill_(-100)
        targets[kept] = whole[kept]
        graph.replay()
        want = _backward(hidden, weight, targets, lse, None, 0.5, dht, BF16)
        assert torch.equal(dh, want[0]) and torch.equal(dw, want[1]), n
        _check_backward(hidden, weight, targets, lse, dh, dw, None, 0.5)


# ---- head loss: logits that overflow, and parts of the vocabulary that are far below the rest --------------

@pytest.mark.parametrize("dht", [BF16, F32])
@pytest.mark.parametrize("below", [[(0, 16)], [(128, 144)], [(0, 128)], [(256, 512)], [(0, 16), (128, 256), (384, 500)], [(16, 500)], [(1, 500)]])
def test_head_loss_where_logits_are_minus_infinity(below, dht):
    """Products of -1e20 and 1e20 overflow: those logits are -inf, their tokens' losses are those of the rest of the vocabulary,
    and their weight's rows get no gradient."""
    tokens, vocab, width = 70, 500, 64
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width)
    hidden[:, 0], weight[:, 0] = 1e20, 0
    rest = torch.ones(vocab, dtype=torch.bool, device="cuda")
    for a, b in below:
        weight[a:b] = 0
        weight[a:b, 0] = -1e20
        rest[a:b] = False
    left = rest.nonzero()[:, 0]
    targets = left[torch.randint(0, len(left), (tokens,), generator=_gen(3), device="cuda")]
    loss, lse = _forward(hidden, weight, targets)
    h, w = hidden.clone(), weight[left]
    h[:, 0] = 0                                          # (times a column of zeros)
    place = torch.searchsorted(left, targets)
    _check_forward(h, w, place, loss, lse)
    lse = R.head_loss(h, w, place)[1].float()
    dh, dw = _backward(hidden, weight, targets, lse, None, 1.0, dht, BF16)
    assert (dw[~rest] == 0).all()
    # column 0 apart: there a gradient of (about) nothing meets 1e20
    _check_backward(h[:, 1:].contiguous(), w[:, 1:].contiguous(), place, lse, dh[:, 1:], dw[left][:, 1:])


@pytest.mark.parametrize("low", [(0, 16), (128, 144), (256, 300), (384, 500), (0, 128)])
def test_head_loss_where_the_first_logits_of_a_part_are_far_below_the_rest(low):
    """The sum of exponentials starts from the greatest of 16 logits; here the others are up to 2^184 times larger."""
    tokens, vocab, width = 70, 500, 64
    hidden, _, weight, _, targets = _head_case(tokens, vocab, width)
    hidden[:, 0], weight[:, 0] = 8, 0
    weight[low[0]:low[1], 0] = -16
    loss, lse = _forward(hidden, weight, targets, label_smoothing=0.1)
    _check_forward(hidden, weight, targets, loss, lse, smooth=0.1)
    dh, dw = _backward(hidden, weight, targets, lse, None, 1.0, F32, F32, label_smoothing=0.1)
    _check_backward(hidden, weight, targets, lse, dh, dw, smooth=0.1)


# ---- matrices side by side in one buffer ------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,ld", [(7, 64, 128), (5, 33, 66), (300, 1601, 3202), (9, 40, 96), (4, 9000, 18000)])
def test_operators_on_columns_of_one_buffer(dtype, rows, cols, ld):
    """x and y as neighbouring columns of one matrix: they share no element."""
    g = _gen(rows)
    buf = torch.randn(rows, ld, generator=g, device="cuda").to(dtype)
    x, y = buf[:, :cols], buf[:, cols:2 * cols]
    behind = buf[:, 2 * cols:].clone()
    xs, r = x.contiguous(), torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    want = torch.empty_like(xs)
    A.adapm_dropout(xs, r, want, TYPE[dtype], rows, cols, 0.3, 1, 2)
    A.adapm_dropout(x, r, y, TYPE[dtype], rows, cols, 0.3, 1, 2, x_ld=ld, y_ld=ld)
    assert torch.equal(y, want) and torch.equal(x, xs) and torch.equal(buf[:, 2 * cols:], behind)
    w = torch.randn(cols, generator=g, device="cuda").to(dtype)
    rstd, again = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    A.adapm_rmsnorm_forward(A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype]), xs, None, w, None, want, None, None, rstd)
    A.adapm_rmsnorm_forward(A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], x_ld=ld, y_ld=ld), x, None, w, None, y, None, None, again)
    _close(y, want.double(), want.double().abs() * (2 * HALF[dtype] + 2.0**-16), "y")          # (another layout may take another order of the sum)
    _close(again, rstd.double(), rstd.double() * 2.0**-16, "rstd")
    assert torch.equal(x, xs) and torch.equal(buf[:, 2 * cols:], behind)
    dy = torch.randn(rows, cols, generator=g, device="cuda").to(dtype)
    A.adapm_rmsnorm_backward(A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype]), dy, None, xs, rstd, w, want, None, None, A.TYPE_F32, False, None)
    A.adapm_rmsnorm_backward(A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], sum_ld=ld, residual_ld=ld), dy, None, x, rstd, w, y, None, None, A.TYPE_F32, False, None)
    size = (rstd[:, None] * (dy.float() * w.float()).abs()).double()
    _close(y, want.double(), want.double().abs() * 2 * HALF[dtype] + (size + size.amax(1, keepdim=True)) * 2.0**-16 * (1 + x.double().abs()), "dresidual")
    assert torch.equal(x, xs) and torch.equal(buf[:, 2 * cols:], behind)


def test_head_gradients_beside_their_operands():
    """dhidden in the columns beside hidden's, dweight in those beside the weight's."""
    hidden, _, weight, _, targets = _head_case(300, 1000, 64, ignored=0.2)
    lse = R.head_loss(hidden, weight, targets)[1].float()
    dh, dw = _backward(hidden, weight, targets, lse)
    hb, wb = torch.full((300, 136), GUARD, dtype=BF16, device="cuda"), torch.full((1000, 128), GUARD, dtype=BF16, device="cuda")
    hb[:, :64], wb[:, 64:] = hidden, weight
    d = A.head_loss_desc(300, 1000, 64, 136, 128)
    scratch = torch.empty(A.adapm_head_loss_scratch_bytes(d, True), dtype=torch.uint8, device="cuda")
    A.adapm_head_loss_backward(d, hb, wb[:, 64:], targets, lse, None, 1.0, hb[:, 64:], wb, scratch)
    assert torch.equal(hb[:, 64:128], dh) and torch.equal(wb[:, :64], dw)
    assert torch.equal(hb[:, :64].nan_to_num(3), hidden.nan_to_num(3)) and torch.equal(wb[:, 64:], weight) and (hb[:, 128:] == GUARD).all()


def test_head_gradients_directly_behind_a_view_of_their_operands():
    """hidden as columns of a wider matrix whose last row ends before its pitch does: what follows may be an output."""
    hidden, _, weight, _, targets = _head_case(40, 300, 64)
    lse = R.head_loss(hidden, weight, targets)[1].float()
    dh, _ = _backward(hidden, weight, targets, lse)
    arena = torch.full((39 * 128 + 64 + 39 * 128 + 64,), GUARD, dtype=BF16, device="cuda")
    h, out = arena[:39 * 128 + 64].as_strided((40, 64), (128, 1)), arena.as_strided((40, 64), (128, 1), 39 * 128 + 64)
    h.copy_(hidden)
    d = A.head_loss_desc(40, 300, 64, 128)
    scratch = torch.empty(A.adapm_head_loss_scratch_bytes(d, True), dtype=torch.uint8, device="cuda")
    A.adapm_head_loss_backward(d, h, weight, targets, lse, None, 1.0, out, None, scratch)
    assert torch.equal(out, dh) and torch.equal(h, hidden)


# ---- RMS norm: every form of its kernels with the branch's dropout ----------------------------------------

DROP_SIZES = [  # rows, cols, pitch added, shift of the buffers in elements
    (2400, 64, 0, 0), (2400, 248, 8, 0), (2400, 512, 0, 0), (2371, 1024, 0, 0), (2369, 1600, 0, 0), (9, 1600, 0, 0), (9, 9000, 0, 0), (5, 20000, 8, 0),
    (2400, 333, 0, 1), (7, 9000, 0, 1), (2400, 1001, 0, 0), (2400, 255, 0, 8), (20, 1001, 0, 0), (9, 9001, 0, 0), (2400, 769, 0, 0),
    (1200, 8195, 0, 0), (1300, 2056, 3, 0), (5000, 41, 0, 0),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,pad,shift", DROP_SIZES)
def test_rmsnorm_with_dropout_in_every_form(dtype, rows, cols, pad, shift):
    g = _gen(rows + 5 * cols)
    ld = cols + pad
    x, xb = _rows(g, rows, cols, dtype, ld, shift)
    r, _ = _rows(g, rows, cols, dtype, ld + 8, shift, std=3.0)
    w = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(dtype)
    p, seed, offset = 0.25, 0x77_12345678, (1 << 33) + 6
    keep = R.keep_mask_wide(rows, cols, p, seed, offset, "cuda")
    x[~keep] = float("nan")                            # what is dropped reaches nothing
    (s, sb), (y, yb) = (_rows(g, rows, cols, dtype, ld, shift, 0.0) for _ in range(2))
    rstd = torch.empty(rows, device="cuda")
    d = A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], 1e-5, drop_p=p, seed=seed, offset=offset, x_ld=ld, residual_ld=ld + 8, sum_ld=ld, y_ld=ld)
    A.adapm_rmsnorm_forward(d, x, r, w, s, y, None, None, rstd)
    ws, wr, wy = R.rmsnorm(x, r, w, 1e-5, keep, p)
    fp = (64 + 15 + 8) * 2.0**-24
    most = R.drop(x.double(), keep, p).abs() + r.double().abs()          # the product and the sum are rounded to fp32 before the last rounding
    sums = (most.square().sum(1) / ws.square().sum(1)).sqrt()
    _close(s, ws, ws.abs() * HALF[dtype] * 1.01 + most * 2.0**-23, "sum")
    _close(rstd, wr, wr * (fp + sums * 2.0**-22), "rstd")
    _close(y, wy, wy.abs() * (HALF[dtype] * 1.01 + fp + sums[:, None] * 2.0**-22 + 2.0**-22) + most * 2.0**-22 * wr[:, None] * w.double().abs(), "y")
    for m, b in ((s, sb), (y, yb)):
        T._guards_stand(m, b)
    # its gradient: the same mask
    dy, _ = _rows(g, rows, cols, dtype, ld, shift)
    dsum, _ = _rows(g, rows, cols, dtype, ld, shift)
    (dres, db), (dx, dxb) = _rows(g, rows, cols, dtype, ld + 8, shift, 0.0), _rows(g, rows, cols, dtype, ld, shift, 0.0)
    dw = torch.empty(cols, device="cuda")
    scratch = torch.empty(A.adapm_rmsnorm_backward_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    A.adapm_rmsnorm_backward(d, dy, dsum, s, rstd, w, dres, dx, dw, A.TYPE_F32, False, scratch)
    want, wdx, wdw = R.rmsnorm_grad(dy, dsum, s, rstd, w, keep, p)
    xh, dyw = s.double() * rstd.double()[:, None], dy.double() * w.double()
    inner = (dyw * xh).abs().mean(1, keepdim=True)
    bound = rstd.double()[:, None] * (dyw.abs() * 2.0**-21 + xh.abs() * inner * (fp + 2.0**-21)) + dsum.double().abs() * 2.0**-23
    _close(dres, want, bound + want.abs() * HALF[dtype] * 1.01, "dresidual")
    _close(dx, wdx, 4 / 3 * bound * 1.01 + wdx.abs() * (HALF[dtype] * 1.01 + 2.0**-22), "dx")
    assert (dx[~keep] == 0).all()
    _close(dw, wdw, (dy.double() * xh).abs().sum(0) * ((rows / 100 + 64 + 8) * 2.0**-24), "dweight")
    for m, b in ((dres, db), (dx, dxb)):
        T._guards_stand(m, b)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,shift", [(2400, 512, 0), (2369, 1600, 0), (9, 9000, 0), (5, 1000, 1), (2400, 1001, 0)])
@pytest.mark.parametrize("group", [0, 128])
def test_rmsnorm_with_dropout_in_8_bits(dtype, rows, cols, shift, group):
    """The scales and values are those of y as the plain form has it."""
    g = _gen(rows * 3 + cols)
    x, _ = _rows(g, rows, cols, dtype, cols, shift)
    r, _ = _rows(g, rows, cols, dtype, cols, shift)
    w = torch.ones(cols, dtype=dtype, device="cuda")
    keep = R.keep_mask_wide(rows, cols, 0.1, 3, 4, "cuda")
    q, scales = torch.empty(rows, cols, dtype=torch.uint8, device="cuda"), torch.empty(rows, -(-cols // group) if group else 1, device="cuda")
    A.adapm_rmsnorm_forward(A.rmsnorm_desc(rows, cols, TYPE[dtype], TYPE[dtype], 1e-5, drop_p=0.1, seed=3, offset=4, q8_group=group),
                            x, r, w, None, None, q, scales, None)
    ws, wr, wy = R.rmsnorm(x, r, w, 1e-5, keep, 0.1)
    most = R.drop(x.double(), keep, 0.1).abs() + r.double().abs()
    sums = (most.square().sum(1) / ws.square().sum(1)).sqrt()[:, None]
    fp = (64 + 15 + 8) * 2.0**-24 + 2.0**-21 + sums * 2.0**-22
    want = R.quantize_scales(wy, group)
    absolute = most * 2.0**-22 * wr[:, None]
    per = scales.double().repeat_interleave(group or cols, 1)[:, :cols]
    _close(scales, want, want * fp + absolute.amax(1, keepdim=True) / 448, "scales")
    # e4m3: half a step is 2^-4 of the value, and 2^-10 below the smallest normal number
    _close(q.view(torch.float8_e4m3fn).double() * per, wy, wy.abs() * (2.0**-4 + 2 * fp) + per * 2.0**-10 + 2 * absolute.amax(1, keepdim=True), "y8")
