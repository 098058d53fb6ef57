"""Plain 64-bit forms of the operators around the step: dropout, RMS norm, the head's loss, and their gradients.

Written from the definitions in include/adapm.h, on torch tensors in fp64 of any device.  Test infrastructure only; shares
no code with the library.
"""
from __future__ import annotations

import torch


# ---- dropout -------------------------------------------------------------------------------------------

def philox4x32_10(counter, key):
    """One block of Philox4x32 with ten rounds on Python integers (Salmon et al., SC 2011): four 32-bit words."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def least_kept(p: float) -> int:
    return round(p * 65536)


def keep_mask(rows: int, cols: int, p: float, seed: int, offset: int) -> torch.Tensor:
    """Which elements dropout keeps, element by element (small sizes: a Python loop)."""
    groups = (cols + 7) // 8
    mask = torch.zeros(rows, cols, dtype=torch.bool)
    low = 0xFFFFFFFF
    for r in range(rows):
        for g in range(groups):
            q = r * groups + g
            w = philox4x32_10((q & low, q >> 32, offset & low, offset >> 32), (seed & low, seed >> 32))
            for j in range(min(8, cols - 8 * g)):
                mask[r, 8 * g + j] = ((w[j // 2] >> (16 * (j % 2))) & 0xFFFF) >= least_kept(p)
    return mask


def keep_mask_wide(rows: int, cols: int, p: float, seed: int, offset: int, device="cpu") -> torch.Tensor:
    """The same for large sizes: all counters at once in 64-bit tensors, whose products keep the lower 64 bits."""
    low, groups = 0xFFFFFFFF, (cols + 7) // 8
    q = torch.arange(rows * groups, device=device)
    c = [q & low, q >> 32, torch.full_like(q, offset & low), torch.full_like(q, offset >> 32)]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) & low ^ c[1] ^ k[0], b & low, (a >> 32) & low ^ c[3] ^ k[1], a & low]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    halves = torch.stack([c[j // 2] >> (16 * (j % 2)) & 0xFFFF for j in range(8)], 1)
    return halves.view(rows, 8 * groups)[:, :cols] >= least_kept(p)


def drop(x: torch.Tensor, keep, p: float) -> torch.Tensor:
    least = least_kept(p)
    if least == 0:
        return x
    return torch.where(keep, x * (65536 / (65536 - least) if least < 65536 else 0.0), torch.zeros_like(x))


# ---- RMS norm ------------------------------------------------------------------------------------------

def rmsnorm(x, residual, weight, eps, keep=None, p=0.0):
    """(s, rstd, y) in fp64."""
    s = x.double() if keep is None else drop(x.double(), keep, p)
    if residual is not None:
        s = s + residual.double()
    rstd = 1 / (s.square().mean(1) + eps).sqrt()
    return s, rstd, s * rstd[:, None] * weight.double()


def quantize_scales(y, group):
    """Scales of the 8-bit output: m / 448 per row (group 0) or per group of columns, 1 where m is 0."""
    parts = y.split(group or y.shape[1], 1)
    m = torch.stack([t.abs().amax(1) for t in parts], 1)
    return torch.where(m > 0, m / 448, torch.ones_like(m))


def rmsnorm_grad(dy, dsum, s, rstd, weight, keep=None, p=0.0):
    """(dresidual, dx, dweight) in fp64, from the stored s and rstd."""
    dy, s, r, w = dy.double(), s.double(), rstd.double()[:, None], weight.double()
    xh = s * r
    ds = r * (dy * w - xh * (dy * w * xh).mean(1, keepdim=True))
    if dsum is not None:
        ds = ds + dsum.double()
    return ds, (ds if keep is None else drop(ds, keep, p)), (dy * xh).sum(0)


# ---- head loss -----------------------------------------------------------------------------------------

def valid_targets(targets, vocab, ignore):
    return (targets != ignore) & (targets >= 0) & (targets < vocab)


def head_loss(hidden, weight, targets, ignore=-100, smooth=0.0, z_loss=0.0):
    """(loss, lse) per token in fp64: 0 for ignored tokens, NaN for other targets out of range."""
    vocab = weight.shape[0]
    valid = valid_targets(targets, vocab, ignore)
    loss = torch.zeros(len(targets), dtype=torch.float64, device=hidden.device)
    loss[(targets != ignore) & ~valid] = float("nan")
    lse = loss.clone()
    z = hidden[valid].double() @ weight.double().T
    y = targets[valid]
    l = torch.logsumexp(z, 1) if len(y) else z.sum(1)
    lse[valid] = l
    loss[valid] = l - (1 - smooth) * z.gather(1, y[:, None])[:, 0] - smooth * z.mean(1) + z_loss * l * l
    return loss, lse


def head_logit_grad(hidden, weight, targets, lse, dloss=None, scale=1.0, ignore=-100, smooth=0.0, z_loss=0.0):
    """(indices of the valid tokens, gradient of scale * sum(dloss * loss) with respect to their logits), in fp64."""
    vocab = weight.shape[0]
    at = valid_targets(targets, vocab, ignore).nonzero()[:, 0]
    l = lse[at].double()[:, None]
    g = torch.exp(hidden[at].double() @ weight.double().T - l) * (1 + 2 * z_loss * l) - smooth / vocab
    g[torch.arange(len(at), device=g.device), targets[at]] -= 1 - smooth
    if dloss is not None:
        g = g * dloss[at].double()[:, None]
    return at, scale * g


def head_loss_grad(hidden, weight, targets, lse, dloss=None, scale=1.0, ignore=-100, smooth=0.0, z_loss=0.0):
    """(dhidden, dweight) in fp64."""
    at, g = head_logit_grad(hidden, weight, targets, lse, dloss, scale, ignore, smooth, z_loss)
    dh = torch.zeros(hidden.shape, dtype=torch.float64, device=hidden.device)
    dh[at] = g @ weight.double()
    return dh, g.T @ hidden[at].double()
