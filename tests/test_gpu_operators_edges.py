"""Dropout, the RMS norm and the head loss on a GPU at calls that the documentation allows and that lie between the cases of
test_gpu_operators.py, whose helpers and derivations these use."""
import pytest

import test_gpu_operators as T
from oracle import operators_oracle as R
from test_gpu_operators import BF16, F32, HALF, _backward, _check_backward, _close, _gen, _head_case

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
