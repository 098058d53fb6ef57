"""Linear layers in 8 bits on a GPU at calls that the documentation allows and that lie between the cases of test_gpu_linear8.py, whose helpers
and derivations these use; and a layer's training step of several calls, into the optimizer's step."""
import pytest

import paper_2510_09103_b200 as A
import test_gpu_linear8 as T
from oracle import linear8_oracle as R
from test_gpu_operators import BF16, F32, HALF, TYPE, _close, _gen, _rows

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

EINVAL = -1


def _weights(g, out, inn):
    return T._codes(g, out, inn), T._scales(g, out, pow2=False)


# ---- what must not reach what ----------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,out,inn", [(5, 200, 256), (300, 520, 384), (3000, 2056, 512)])
def test_scales_that_are_nan_stay_in_their_rows_and_columns(tokens, out, inn):
    g = _gen(1)
    x8, w8, xs, ws = T._codes(g, tokens, inn), T._codes(g, out, inn), T._scales(g, tokens), T._scales(g, out)
    good = T._run_forward(x8, xs, w8, ws)
    xs2, ws2 = xs.clone(), ws.clone()
    xs2[tokens // 2], ws2[out - 1] = float("nan"), float("inf")
    y = T._run_forward(x8, xs2, w8, ws2)
    assert y[tokens // 2].isnan().all() and not y[:, out - 1].isfinite().any()
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[tokens // 2], keep[:, out - 1] = False, False
    assert torch.equal(y[keep], good[keep])


@pytest.mark.parametrize("tokens,out,inn", [(5, 200, 384), (300, 520, 384), (1500, 2056, 1024)])
def test_gradients_that_are_not_finite_stay_in_their_rows(tokens, out, inn):
    g = _gen(2)
    dy, _ = _rows(g, tokens, out, BF16)
    w8, ws = _weights(g, out, inn)
    x8, xs = T._codes(g, tokens, inn), T._scales(g, tokens, 1 + (inn - 1) // 128)
    dx, dw = T._run_input_grad(dy, w8, ws), T._run_weight_grad(dy, x8, xs, "int8", 128)
    bad = dy.clone()
    bad[tokens - 1, 3] = float("nan")
    dx2, dw2 = T._run_input_grad(bad, w8, ws), T._run_weight_grad(bad, x8, xs, "int8", 128)
    assert dx2[-1].isnan().all() and torch.equal(dx2[:-1], dx[:-1])
    assert dw2[3].isnan().all() and torch.equal(dw2[:3], dw[:3]) and torch.equal(dw2[4:], dw[4:])
    xs[0, 1] = float("nan")                                          # 128 columns of one token
    dw3 = T._run_weight_grad(dy, x8, xs, "int8", 128)
    assert dw3[:, 128:256].isnan().all() and torch.equal(dw3[:, :128], dw[:, :128]) and torch.equal(dw3[:, 256:], dw[:, 256:])


@pytest.mark.parametrize("tokens", [1, 37, 300, 1100])
def test_rows_behind_the_last_token_are_not_read_nor_written(tokens):
    """A padded batch: what lies behind its tokens holds NaN scales, NaN gradients and codes."""
    g = _gen(3)
    out, inn, more = 1032, 264, 300
    x8, w8 = T._codes(g, tokens + more, inn), T._codes(g, out, inn)
    xs, ws = T._scales(g, tokens + more), T._scales(g, out)
    dy, _ = _rows(g, tokens + more, out, BF16)
    xs[tokens:], dy[tokens:] = float("nan"), float("nan")
    y = torch.full((tokens + more, out), 7.0, dtype=BF16, device="cuda")
    dx = torch.full((tokens + more, inn), 7.0, dtype=BF16, device="cuda")
    d = A.linear8_desc(tokens, out, inn, x8_ld=x8.stride(0), w8_ld=w8.stride(0))
    dw = torch.empty(out, inn, dtype=BF16, device="cuda")
    A.adapm_linear8_forward(d, x8, xs, w8, ws, y, T._scratch(d, A.LINEAR8_FORWARD))
    A.adapm_linear8_input_grad(d, dy, w8, ws, dx, T._scratch(d, A.LINEAR8_INPUT_GRAD))
    A.adapm_linear8_weight_grad(d, dy, x8, xs, dw, T._scratch(d, A.LINEAR8_WEIGHT_GRAD))
    assert (y[tokens:] == 7).all() and (dx[tokens:] == 7).all()
    assert torch.equal(y[:tokens], T._run_forward(x8[:tokens], xs[:tokens], w8, ws))
    assert torch.equal(dx[:tokens], T._run_input_grad(dy[:tokens], w8, ws))
    assert torch.equal(dw, T._run_weight_grad(dy[:tokens], x8[:tokens], xs[:tokens, None], "int8", 0)) and dw.isfinite().all()


def test_no_token():
    g = _gen(4)
    w8, ws = _weights(g, 64, 96)
    d = A.linear8_desc(0, 64, 96, w8_ld=w8.stride(0))
    empty = torch.empty(0, 64, device="cuda", dtype=BF16)
    A.adapm_linear8_forward(d, empty, empty, w8, ws, empty, None)
    A.adapm_linear8_input_grad(d, empty, w8, ws, empty, None)
    for dtype in (BF16, F32):
        dw, buf = _rows(None, 64, 96, dtype, 104, 0, 3.0)
        A.adapm_linear8_weight_grad(A.linear8_desc(0, 64, 96, dweight_dtype=TYPE[dtype], dweight_ld=104), empty, empty, empty, dw, None)
        assert (dw == 0).all()
        T._guards_stand(dw, buf)
        dw.fill_(3.0)
        A.adapm_linear8_weight_grad(A.linear8_desc(0, 64, 96, dweight_dtype=TYPE[dtype], dweight_ld=104, accumulate=True), empty, empty, empty, dw, None)
        assert (dw == 3).all()
    A.adapm_quant8(A.quant8_desc(0, 96), None, None, None)
    A.adapm_dequant8(A.quant8_desc(0, 96), None, None, None)


def test_the_largest_sums_of_codes():
    """All codes -128 over the longest K: the sum is 2^30, with fp32 scales that bring it back."""
    inn = 65536
    x8 = torch.full((3, inn), -128, dtype=torch.int8, device="cuda")
    w8 = torch.full((136, inn), -128, dtype=torch.int8, device="cuda")
    w8[7] = 127
    ones = torch.ones(136, device="cuda")
    y = T._run_forward(x8, ones[:3], w8, ones, F32)
    want = torch.full((3, 136), 2.0**30, device="cuda")
    want[:, 7] = -128 * 127 * 65536
    assert torch.equal(y, want)


# ---- long sums, large matrices -----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weight_grad_of_a_long_batch_in_one_piece(dtype):
    """More stages of K than one accumulator takes, and tiles enough that K is not cut: sums in segments.  All products have one
    sign, so that what the tensor cores cut off would add up."""
    tokens, out, inn = 17000, 4096, 2560
    g = _gen(5)
    dy = torch.rand(tokens, out, generator=g, device="cuda").to(BF16)
    x8 = torch.randint(0, 128, (tokens, inn), generator=g, device="cuda").to(torch.int8)
    xs = T._scales(g, tokens, 1)
    dw = T._run_weight_grad(dy, x8, xs, "int8", 0, dtype)
    at = torch.arange(0, out, 97, device="cuda")
    want = dy[:, at].double().T @ R.decode(x8, xs, 0)
    _close(dw[at], want, want * (T._tensor_sum(tokens, 256 if dtype == F32 else 4096) + HALF[dtype] * 1.01), "dweight")


def test_results_past_32_bits_of_elements():
    g = _gen(6)
    tokens, out, inn = 70000, 32768, 16
    x8, xs = T._codes(g, tokens, inn), T._scales(g, tokens)
    w8, ws = _weights(g, out, inn)
    d = A.linear8_desc(tokens, out, inn)
    y = torch.empty(tokens, out, dtype=BF16, device="cuda")
    A.adapm_linear8_forward(d, x8, xs, w8, ws, y, T._scratch(d, A.LINEAR8_FORWARD))
    at = torch.tensor([0, 65534, 65535, 65536, 69999], device="cuda")
    want = R.forward(x8[at].view(torch.int8), xs[at], w8.view(torch.int8), ws)
    _close(y[at], want, want.abs() * (3.1 * 2.0**-24 + HALF[BF16] * 1.01) + 1e-37, "y")
    # the same matrix as dy: offsets of the operand
    dx = torch.empty(tokens, inn, dtype=BF16, device="cuda")
    A.adapm_linear8_input_grad(d, y, w8, ws, dx, T._scratch(d, A.LINEAR8_INPUT_GRAD))
    w = R.decode(w8.view(torch.int8), ws, 0)
    want, size = y[at].double() @ w, y[at].double().abs() @ w.abs()
    _close(dx[at], want, T._bound(size, want, out, BF16, False), "dx")
    dw = torch.empty(out, inn, dtype=BF16, device="cuda")
    A.adapm_linear8_weight_grad(d, y, x8, xs, dw, T._scratch(d, A.LINEAR8_WEIGHT_GRAD))
    rows = torch.tensor([0, 1, 16384, 32766, 32767], device="cuda")
    x = R.decode(x8.view(torch.int8), xs, 0)
    want, size = y[:, rows].double().T @ x, y[:, rows].double().abs().T @ x.abs()
    _close(dw[rows], want, T._bound(size, want, tokens, BF16, True), "dweight")


def test_the_largest_weight_gradient():
    g = _gen(7)
    out = inn = 65536
    dy = torch.randn(2, out, generator=g, device="cuda").to(BF16)
    x8, xs = T._codes(g, 2, inn), T._scales(g, 2, inn // 128)
    d = A.linear8_desc(2, out, inn, x_group=128)
    dw = torch.empty(out, inn, dtype=BF16, device="cuda")
    A.adapm_linear8_weight_grad(d, dy, x8, xs, dw, T._scratch(d, A.LINEAR8_WEIGHT_GRAD))
    x = R.decode(x8.view(torch.int8), xs, 128)
    for at in (slice(0, 64), slice(32760, 32780), slice(out - 64, out)):
        want = dy[:, at].double().T @ x
        _close(dw[at], want, T._bound(dy[:, at].double().abs().T @ x.abs(), want, 2, BF16, True), "dweight")


# ---- streams, graphs, repeated calls -------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,out,inn", [(3, 640, 512), (200, 1376, 512), (1100, 1024, 1032)])
def test_calls_on_other_streams_in_graphs_and_again_give_the_same_bits(tokens, out, inn):
    g = _gen(8)
    x, _ = _rows(g, tokens, inn, BF16)
    w, _ = _rows(g, out, inn, BF16, std=0.02)
    dy, _ = _rows(g, tokens, out, BF16)

    def buffers():
        ld = -(-inn // 16) * 16
        d = A.linear8_desc(tokens, out, inn, x8_ld=ld, w8_ld=ld)
        new = lambda *s: torch.empty(*s, dtype=BF16, device="cuda")  # noqa: E731
        return dict(d=d, ld=ld, x8=torch.empty(tokens, ld, dtype=torch.int8, device="cuda"), w8=torch.empty(out, ld, dtype=torch.int8, device="cuda"),
                    xs=torch.empty(tokens, device="cuda"), ws=torch.empty(out, device="cuda"), y=new(tokens, out), dx=new(tokens, inn), dw=new(out, inn),
                    scratch=[T._scratch(d, i) for i in range(3)])

    def run(b):
        A.adapm_quant8(A.quant8_desc(tokens, inn, codes_ld=b["ld"]), x, b["x8"], b["xs"])
        A.adapm_quant8(A.quant8_desc(out, inn, codes_ld=b["ld"]), w, b["w8"], b["ws"])
        A.adapm_linear8_forward(b["d"], b["x8"], b["xs"], b["w8"], b["ws"], b["y"], b["scratch"][0])
        A.adapm_linear8_input_grad(b["d"], dy, b["w8"], b["ws"], b["dx"], b["scratch"][1])
        A.adapm_linear8_weight_grad(b["d"], dy, b["x8"], b["xs"], b["dw"], b["scratch"][2])

    first, side, graphed, second = buffers(), buffers(), buffers(), buffers()
    run(first)
    want = {k: first[k].clone() for k in ("y", "dx", "dw")}
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):                      # two calls at once, each with its own scratch
        for _ in range(5):
            run(side)
    for _ in range(5):
        run(second)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(graphed)
    for _ in range(3):
        for k in want:
            graphed[k].fill_(5)
        graph.replay()
    torch.cuda.synchronize()
    for b in (side, second, graphed):
        for k in want:
            assert torch.equal(b[k], want[k]), k
        assert all(A.adapm_linear8_status(s) == 0 for s in b["scratch"])


def test_memory_of_the_host_is_refused():
    host = torch.zeros(64, 64, dtype=torch.int8).pin_memory()
    there = torch.zeros(64, 64, dtype=torch.int8, device="cuda")
    ones, wide = torch.ones(64, device="cuda"), torch.empty(64, 64, dtype=BF16, device="cuda")
    d, q = A.linear8_desc(64, 64, 64), A.quant8_desc(64, 64)
    for call in (lambda: A.adapm_quant8(q, wide, host, ones), lambda: A.adapm_dequant8(q, host, ones, wide),
                 lambda: A.adapm_linear8_forward(d, host, ones, there, ones, wide, T._scratch(d, 0)),
                 lambda: A.adapm_linear8_input_grad(d, wide, host, ones, torch.empty_like(wide), T._scratch(d, 1)),
                 lambda: A.adapm_linear8_weight_grad(d, wide, there, ones, host.view(torch.uint8).repeat(1, 2), T._scratch(d, 2))):
        with pytest.raises(A.AdapmError) as e:
            call()
        assert e.value.code == EINVAL


# ---- together ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens", [40, 700])
def test_a_layer_in_8_bits_between_the_norm_and_the_step(tokens):
    """The norm's output to 8 bits, through the weight that the step keeps in bf16, back into the gradients that the step reads: every
    number against the 64-bit forms, and the gradients against differences of the layer's own function."""
    out, inn = 264, 192
    g = _gen(9)
    blocks = [A.adapm_block(0, out, inn, A.MOM_FULL, 0, A.V_ELEMENT, 1, 1.0, 0.0)]
    ctx = A.adapm_create(blocks, A.hparams(lr=1e-2, grad_dtype=A.GRAD_BF16))
    params = torch.randn(out * inn, generator=g, device="cuda") * 0.05
    grads = torch.zeros(out * inn, dtype=BF16, device="cuda")
    shadow = params.to(BF16)
    state = torch.zeros(max(1, ctx.adapm_state_bytes() // 4), device="cuda")
    work = torch.zeros(max(1, ctx.adapm_workspace_bytes() // 4), device="cuda")
    ctx.adapm_set_workspace(work)
    ctx.adapm_set_shadow_params(shadow)
    ctx.adapm_state_init(state)
    stream, norm_w = torch.randn(tokens, inn, generator=g, device="cuda").to(BF16), torch.ones(inn, dtype=BF16, device="cuda")
    dy = (torch.randn(tokens, out, generator=g, device="cuda") * 1e-2).to(BF16)
    h, y, dh, dstream = (torch.empty(tokens, n, dtype=BF16, device="cuda") for n in (inn, out, inn, inn))
    rstd = torch.empty(tokens, device="cuda")
    x8, w8 = torch.empty(tokens, inn, dtype=torch.int8, device="cuda"), torch.empty(out, inn, dtype=torch.int8, device="cuda")
    xs, ws = torch.empty(tokens, device="cuda"), torch.empty(out, device="cuda")
    nd, d = A.rmsnorm_desc(tokens, inn), A.linear8_desc(tokens, out, inn)
    scratch = [T._scratch(d, i) for i in range(3)]
    norm_scratch = torch.empty(A.adapm_rmsnorm_backward_scratch_bytes(nd), dtype=torch.uint8, device="cuda")
    for t in (1, 2):
        A.adapm_quant8(A.quant8_desc(out, inn, pow2=True), shadow, w8, ws)
        A.adapm_rmsnorm_forward(nd, stream, None, norm_w, None, h, None, None, rstd)
        A.adapm_quant8(A.quant8_desc(tokens, inn, pow2=True), h, x8, xs)
        A.adapm_linear8_forward(d, x8, xs, w8, ws, y, scratch[0])
        A.adapm_linear8_input_grad(d, dy, w8, ws, dh, scratch[1])
        A.adapm_linear8_weight_grad(d, dy, x8, xs, grads, scratch[2])
        A.adapm_rmsnorm_backward(nd, dh, None, stream, rstd, norm_w, dstream, None, None, A.TYPE_F32, False, norm_scratch)
        x, w = R.decode(x8, xs, 0), R.decode(w8, ws, 0)
        assert torch.equal(ws[:, None].double(), R.scales_of(shadow.view(out, inn), "int8", 0, True))
        assert (x - h.double()).abs().max() <= xs.max() / 2 and (w - shadow.view(out, inn).double()).abs().max() <= ws.max() / 2
        want = x @ w.T
        _close(y, want, want.abs() * (3.1 * 2.0**-24 + HALF[BF16] * 1.01) + 1e-37, "y")
        before = params.clone()
        # loss = sum of dy y is linear in x and in w: its differences are the gradients
        dyd = dy.double()
        loss = lambda x, w: (dyd * (x @ w.T)).sum()  # noqa: E731
        for i, j in ((0, 0), (tokens - 1, inn - 1), (tokens // 2, 7)):
            step = torch.zeros_like(x)
            step[i, j] = 0.5
            diff = loss(x + step, w) - loss(x - step, w)
            bound = (dyd[i].abs() @ w[:, j].abs()) * T._tensor_sum(out, 16384) + diff.abs() * HALF[BF16] * 1.01 + 1e-9
            assert (dh[i, j].double() - diff).abs() <= bound
        dw = grads.view(out, inn)
        for i, j in ((0, 0), (out - 1, inn - 1), (100, 7)):
            step = torch.zeros_like(w)
            step[i, j] = 0.5
            diff = loss(x, w + step) - loss(x, w - step)
            bound = (dyd[:, i].abs() @ x[:, j].abs()) * T._tensor_sum(tokens, 16384) + diff.abs() * HALF[BF16] * 1.01 + 1e-9
            assert (dw[i, j].double() - diff).abs() <= bound
        assert dstream.isfinite().all()
        ctx.adapm_step(params, grads, state, t)
        assert ctx.adapm_get_status() == 0 and not torch.equal(params, before) and torch.equal(shadow, params.to(BF16))
    assert all(A.adapm_linear8_status(s) == 0 for s in scratch)


@pytest.mark.parametrize("tokens", [48, 900])
def test_activations_kept_in_e4m3_by_the_norm_make_the_weight_gradient(tokens):
    """The norm's own 8-bit output, whose scales are no powers of two, as the checkpoint: back to numbers, and into the product."""
    out, inn = 136, 256
    g = _gen(10)
    x, w = torch.randn(tokens, inn, generator=g, device="cuda").to(BF16), torch.ones(inn, dtype=BF16, device="cuda")
    dy, _ = _rows(g, tokens, out, BF16)
    for group in (0, 128):
        y8 = torch.empty(tokens, inn, dtype=T.E4M3, device="cuda")
        scales = torch.empty(tokens, inn // group if group else 1, device="cuda")
        A.adapm_rmsnorm_forward(A.rmsnorm_desc(tokens, inn, q8_group=group), x, None, w, None, None, y8, scales, None)
        back = torch.empty(tokens, inn, device="cuda")
        A.adapm_dequant8(A.quant8_desc(tokens, inn, A.TYPE_F32, A.CODE_E4M3, group), y8, scales, back)
        want = R.decode(y8, scales, group)
        _close(back, want, want.abs() * 2.0**-23, "x")
        T._check_weight_grad(dy, y8.view(torch.uint8), scales, "e4m3", group, BF16, False)


FIRST_CALL_IN_A_CAPTURE = """
import torch, paper_2510_09103_b200 as A
bf16, i8 = torch.bfloat16, torch.int8
def buffers(tokens, out, inn):
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(bf16) for s in ((tokens, inn), (out, inn), (tokens, out)))
    d = A.linear8_desc(tokens, out, inn)
    return dict(d=d, x=x, w=w, dy=dy, x8=torch.zeros(tokens, inn, dtype=i8, device="cuda"), w8=torch.zeros(out, inn, dtype=i8, device="cuda"),
                xs=torch.zeros(tokens, device="cuda"), ws=torch.zeros(out, device="cuda"), y=torch.zeros_like(dy), dx=torch.zeros_like(x), dw=torch.zeros_like(w),
                s=[torch.zeros(A.adapm_linear8_scratch_bytes(d, i), dtype=torch.uint8, device="cuda") for i in range(3)])
def run(b):
    A.adapm_quant8(A.quant8_desc(*b["x"].shape), b["x"], b["x8"], b["xs"])
    A.adapm_quant8(A.quant8_desc(*b["w"].shape), b["w"], b["w8"], b["ws"])
    A.adapm_linear8_forward(b["d"], b["x8"], b["xs"], b["w8"], b["ws"], b["y"], b["s"][0])
    A.adapm_linear8_input_grad(b["d"], b["dy"], b["w8"], b["ws"], b["dx"], b["s"][1])
    A.adapm_linear8_weight_grad(b["d"], b["dy"], b["x8"], b["xs"], b["dw"], b["s"][2])
sets = [buffers(1, 256, 512), buffers(40, 1376, 512), buffers(3000, 2048, 1024)]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    for b in sets: run(b)
graph.replay()
torch.cuda.synchronize()
got = [[b[k].clone() for k in ("y", "dx", "dw")] for b in sets]
for b in sets: run(b)
torch.cuda.synchronize()
for b, old in zip(sets, got):
    for k, o in zip(("y", "dx", "dw"), old): assert torch.equal(b[k], o) and o.float().abs().sum() > 0
print("same")
"""


def test_the_first_call_of_a_process_may_be_a_captured_one():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALL_IN_A_CAPTURE], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,out,inn,pad", [(40, 3592, 4104, 0), (40, 3592, 4104, 8), (200, 4096, 4352, 0), (130, 200, 20000, 24)])
def test_added_weight_gradient_of_many_tiles(dtype, tokens, out, inn, pad):
    """Several tiles to every pair of CTAs, rows on and off sectors of 32 bytes, last tiles that end inside: what is there is read while the tile before is
    still on its way out.  Elements that nothing is added to keep their value to the bit."""
    g = _gen(tokens + out + inn + pad)
    dy, _ = _rows(g, tokens, out, BF16, out, 0)
    dy[:, 5] = 0
    x8 = T._codes(g, tokens, inn)
    xs = T._scales(g, tokens, pow2=True)
    before = (torch.randn(out, inn, generator=g, device="cuda") * 30).to(dtype)
    T._check_weight_grad(dy, x8, xs, "int8", 0, dtype, True, pad, before)
    dw = T._run_weight_grad(dy, x8, xs, "int8", 0, dtype, pad, before)
    assert torch.equal(dw[5], before[5])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,out,inn", [(40, 3592, 4104), (40, 72, 200), (600, 520, 392), (3000, 520, 392)])
def test_gradients_added_one_call_behind_the_other(dtype, tokens, out, inn):
    """A call reads what the one before it has written, whether or not the host waits in between."""
    g = _gen(tokens + out)
    dy, _ = _rows(g, tokens, out, BF16, out, 0)
    x8, xs = T._codes(g, tokens, inn), T._scales(g, tokens, pow2=True)
    d = A.linear8_desc(tokens, out, inn, dweight_dtype=TYPE[dtype], accumulate=True, x8_ld=x8.stride(0))
    scratch = torch.empty(A.adapm_linear8_scratch_bytes(d, A.LINEAR8_WEIGHT_GRAD), dtype=torch.uint8, device="cuda")
    got = []
    for wait in (True, False):
        dw = torch.ones(out, inn, dtype=dtype, device="cuda")
        for _ in range(5):
            A.adapm_linear8_weight_grad(d, dy, x8, xs, dw, scratch)
            if wait:
                assert A.adapm_linear8_status(scratch) == 0
        got.append(dw)
    assert torch.equal(*got)
    assert not torch.equal(got[0], torch.ones_like(got[0]))
