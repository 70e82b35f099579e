"""GELU and SiLU and their slopes at single values, far into the tails where they are small: errors relative to the value itself (to the
size of the slope's two terms), as include/grem.h states them, and one rounding to the type."""
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _close(got, want, off, t, what):
    # (below 2^-120 the 32-bit terms leave the normal numbers)
    tol = off + ref.half_step(t) * (want.abs() + off) + ref.least(t) + 2.0 ** -120
    bad = ((got.cpu().double() - want).abs() > tol).flatten()
    assert not bad.any(), f"{what}: {int(bad.sum())} values off"


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_relative_errors_into_the_tails(name, t):
    # one input column, weight 1: z is the input
    z = torch.cat([torch.linspace(-12, 12, 6001), torch.logspace(-6, 0, 200), -torch.logspace(-6, 0, 200)]).to(t).unsqueeze(1)
    w, act = torch.ones((1, 1), dtype=t, device=DEV), {"gelu": B.ACT_GELU, "silu": B.ACT_SILU}[name]
    zd = z.double()
    if name == "gelu":
        step = 2.0 ** (-20 if t == torch.float32 else -16)
        below, density = 0.5 * torch.special.erfc(-zd / 2 ** 0.5), torch.exp(-zd * zd / 2) / (2 * torch.pi) ** 0.5
        want, off = zd * below, step * (zd * below).abs()
        slope, off_slope = below + zd * density, step * (below + (zd * density).abs())
    else:
        step, s = (zd.abs() + 8) * 2.0 ** -23, torch.sigmoid(zd)
        want, off = zd * s, step * (zd * s).abs()
        slope, off_slope = s + zd * s * torch.sigmoid(-zd), step * s * (1 + zd.abs())
    out, pre = B.grem_linear(z.to(DEV), w, act=act, want_pre=True)
    assert torch.equal(pre.cpu(), z)
    _close(out, want, off, t, name)
    dz = B.grem_linear_backward(torch.ones_like(pre), pre, w, act=act, pre=pre, want_params=False)[0]
    _close(dz, slope, off_slope, t, name + "'s slope")
