"""Linear layers in 8 bits on a GPU: numbers at the edges of fp32's range, and the forms of their kernels that the sizes of test_gpu_linear8.py
pass by.  Helpers and derivations are those of that file."""
import pytest

import test_gpu_linear8 as T

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


# ---- codes next to half a step, of the smallest scales -----------------------------------------------------

@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("cols", [128, 127])
def test_codes_next_to_half_a_step_of_scales_whose_half_is_no_fp32_number(group, cols):
    """Scales from 2^-126 to 2^-125, in units of 2^-149: half of an odd one needs a bit that fp32 does not have there."""
    g = T._gen(11)
    rows = 4096
    unit = 2.0**-149
    s = torch.randint(1 << 23, 1 << 24, (rows,), generator=g, device="cuda").double()
    top = (127 * s * unit).float()                                      # its quotient by 127 is s or a neighbour
    s = (top.double() / 127).float().double() / unit
    assert (s == s.round()).all() and (s % 2 == 1).sum() > rows // 4
    codes = torch.randint(-126, 126, (rows, cols - 1), generator=g, device="cuda").double()
    at = (codes + 0.5) * s[:, None]                                     # half a step: a whole number of units, or half of one
    side = torch.randint(0, 2, (rows, cols - 1), generator=g, device="cuda").bool()
    x = torch.cat([top[:, None].double(), torch.where(side, at.floor(), at.ceil()) * unit], 1)
    # (a number of units above 2^24 is rounded to fp32: a neighbour of the middle all the same)
    codes, scales = T._check_quant(x.float(), "int8", group, False)
    assert torch.equal(scales.double(), s[:, None] * unit)
