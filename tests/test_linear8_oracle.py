"""The plain 64-bit forms of the linear layers in 8 bits against their definitions, number by number, and their gradients against differences."""
import math
from fractions import Fraction

import pytest

from oracle import linear8_oracle as R

torch = pytest.importorskip("torch")


def _scale(m, top, pow2):
    """By exact fractions."""
    if m == 0:
        return Fraction(1)
    q = Fraction(m) / top
    if not pow2:
        return max(Fraction(float(torch.tensor(float(m) / top, dtype=torch.float64).float())), Fraction(2) ** -126)
    k = -126
    while Fraction(2) ** k < q:
        k += 1
    return Fraction(2) ** k


@pytest.mark.parametrize("code,top,pow2", [("int8", 127, False), ("int8", 127, True), ("e4m3", 448, True)])
def test_scales_and_codes_by_fractions(code, top, pow2):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(12, 300, generator=g).bfloat16().float()
    x[0, :], x[1, 3], x[2, 5], x[3, 7], x[4, 150], x[5, 2] = 0, 127.0, 254.0, 448.0, 449.0, 126.5
    for group in (0, 128):
        scales = R.scales_of(x, code, group, pow2)
        codes = R.codes_of(x, scales, code, group)
        for r in range(x.shape[0]):
            for i, part in enumerate(x[r].split(group or 300)):
                s = _scale(part.abs().max().item(), top, pow2)
                assert Fraction(scales[r, i].item()) == s
                for j, v in enumerate(part.tolist()):
                    q, c = Fraction(v) / s, codes[r, (group or 0) * i + j].item()
                    assert abs(c) <= top
                    if code == "int8":
                        assert c == round(q)                     # ties to even
                    else:
                        assert c == torch.tensor(float(q)).to(torch.float8_e4m3fn).float().item()


def test_a_group_that_is_not_finite():
    x = torch.ones(2, 256)
    x[0, 200], x[1, 3] = math.inf, math.nan
    s = R.scales_of(x, "int8", 128, True)
    assert s.isnan().tolist() == [[False, True], [True, False]]
    c = R.codes_of(x, s, "int8", 128)
    assert (c[0, 128:] == 0).all() and (c[1, :128] == 0).all() and R.decode(c, s, 128)[0, 128:].isnan().all()


def test_products_by_loops_and_gradients_against_differences():
    g = torch.Generator().manual_seed(2)
    tokens, out, inn = 3, 4, 130
    x8, w8 = torch.randint(-127, 128, (tokens, inn), generator=g), torch.randint(-127, 128, (out, inn), generator=g)
    xs, ws, dy = torch.rand(tokens, 2, generator=g).double(), torch.rand(out, generator=g).double(), torch.randn(tokens, out, generator=g).double()
    y = R.forward(x8, xs[:, 0], w8, ws)
    for t in range(tokens):
        for n in range(out):
            assert y[t, n].item() == pytest.approx(xs[t, 0].item() * ws[n].item() * sum(int(a) * int(b) for a, b in zip(x8[t], w8[n])), rel=1e-12)
    x, w = R.decode(x8, xs, 128), R.decode(w8, ws, 0)
    assert x[1, 127] == x8[1, 127] * xs[1, 0] and x[1, 128] == x8[1, 128] * xs[1, 1]
    x.requires_grad_(), w.requires_grad_()
    (dy * (x @ w.T)).sum().backward()
    assert torch.allclose(R.input_grad(dy, w8, ws), x.grad, rtol=1e-12) and torch.allclose(R.weight_grad(dy, x8, xs, 128), w.grad, rtol=1e-12)
