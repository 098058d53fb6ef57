"""The plain 64-bit forms that the operators' GPU tests compare with, themselves checked: against published numbers, against
torch's own functions in fp64 and against differences."""
import math

import pytest
import torch

from oracle import operators_oracle as R

D = torch.float64


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def test_philox_gives_the_published_numbers():
    """Known answers of the generator's authors (their file of test vectors, philox4x32 with ten rounds)."""
    assert R.philox4x32_10((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert R.philox4x32_10((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert R.philox4x32_10((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == \
        [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_keeps_the_share_it_says():
    """Binomial: five standard deviations either way."""
    for p in (0.1, 0.5):
        n = 64 * 96
        kept = R.keep_mask(64, 96, p, 7, 1).sum().item()
        assert abs(kept - n * (1 - p)) < 5 * math.sqrt(n * p * (1 - p))
    assert R.keep_mask(4, 20, 0.0, 7, 1).all() and not R.keep_mask(4, 20, 1.0, 7, 1).any()
    x = torch.ones(2, 20, dtype=D)
    assert not R.drop(x * float("nan"), R.keep_mask(2, 20, 1.0, 7, 1), 1.0).any()
    assert not torch.equal(R.keep_mask(8, 64, 0.5, 7, 1), R.keep_mask(8, 64, 0.5, 7, 2))


def test_the_mask_made_at_once_is_the_mask_made_element_by_element():
    for rows, cols, p, seed, offset in ((1, 1, 0.5, 0, 0), (7, 33, 0.3, 0x1234567_89ABCDEF, (1 << 40) + 3), (64, 64, 0.1, 2**64 - 1, 2**63 - 1)):
        assert torch.equal(R.keep_mask_wide(rows, cols, p, seed, offset), R.keep_mask(rows, cols, p, seed, offset))
    assert R.keep_mask_wide(4, 20, 0.0, 7, 1).all() and not R.keep_mask_wide(4, 20, 1.0, 7, 1).any()


def test_rmsnorm_is_torchs_and_its_gradient_autograds():
    g = _gen(1)
    x, res, w = torch.randn(5, 37, generator=g, dtype=D), torch.randn(5, 37, generator=g, dtype=D), torch.randn(37, generator=g, dtype=D)
    keep = R.keep_mask(5, 37, 0.3, 11, 5)
    s, rstd, y = R.rmsnorm(x, res, w, 1e-3, keep, 0.3)
    xa, ra, wa = (t.clone().requires_grad_() for t in (x, res, w))
    sa = R.drop(xa, keep, 0.3) + ra
    ya = torch.nn.functional.rms_norm(sa, (37,), wa, 1e-3)
    assert torch.allclose(y, ya, rtol=1e-12, atol=0)
    dy, dsum = torch.randn(5, 37, generator=g, dtype=D), torch.randn(5, 37, generator=g, dtype=D)
    ((ya * dy).sum() + (sa * dsum).sum()).backward()
    for got, want in zip(R.rmsnorm_grad(dy, dsum, s, rstd, w, keep, 0.3), (ra.grad, xa.grad, wa.grad)):
        assert torch.allclose(got, want, rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("smooth", [0.0, 0.2])
def test_head_loss_is_torchs_cross_entropy(smooth):
    g = _gen(2)
    h, w = torch.randn(9, 16, generator=g, dtype=D), torch.randn(21, 16, generator=g, dtype=D)
    t = torch.randint(0, 21, (9,), generator=g)
    t[3] = -100
    loss, lse = R.head_loss(h, w, t, -100, smooth)
    want = torch.nn.functional.cross_entropy(h @ w.T, t, ignore_index=-100, label_smoothing=smooth, reduction="none")
    assert torch.allclose(loss, want, rtol=1e-12, atol=1e-12) and lse[3] == 0
    t[4] = 21
    assert R.head_loss(h, w, t)[0][4].isnan()


def test_head_loss_gradient_is_autograds_and_the_differences():
    g = _gen(3)
    h, w = torch.randn(6, 8, generator=g, dtype=D), torch.randn(13, 8, generator=g, dtype=D)
    t = torch.randint(0, 13, (6,), generator=g)
    t[0] = -100
    dloss = torch.rand(6, generator=g, dtype=D)

    def total(h, w):
        return 0.7 * (dloss * R.head_loss(h, w, t, -100, 0.1, 0.05)[0]).sum()

    dh, dw = R.head_loss_grad(h, w, t, R.head_loss(h, w, t, -100, 0.1, 0.05)[1], dloss, 0.7, -100, 0.1, 0.05)
    ha, wa = h.clone().requires_grad_(), w.clone().requires_grad_()
    z = ha @ wa.T
    l = torch.logsumexp(z, 1)
    per = torch.nn.functional.cross_entropy(z, t, ignore_index=-100, label_smoothing=0.1, reduction="none") + 0.05 * l * l * (t != -100)
    (0.7 * dloss * per).sum().backward()
    assert torch.allclose(dh, ha.grad, atol=1e-12) and torch.allclose(dw, wa.grad, atol=1e-12)
    # central differences: off by step^2 times a third derivative (of order one), and by rounding / step
    for _ in range(5):
        a, b = torch.randn(h.shape, generator=g, dtype=D), torch.randn(w.shape, generator=g, dtype=D)
        e = 1e-5
        diff = (total(h + e * a, w + e * b) - total(h - e * a, w - e * b)) / (2 * e)
        assert abs(diff - (dh * a).sum() - (dw * b).sum()) < 1e-7
