"""Dropout, the RMS norm and the head loss on a GPU at calls that the documentation allows and that lie between the cases of
test_gpu_operators.py, whose helpers and derivations these use."""
import pytest

from oracle import operators_oracle as R
from test_gpu_operators import BF16, _backward, _check_backward, _head_case

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
