"""Layer norm's backward pass over so many rows that a workgroup takes several in turn.  Given statistics of 0 and 1 and whole numbers, the
parameters' gradients are sums of whole numbers below 2^24: exact in 32 bits in whatever order, so that a row that is lost or taken twice
is seen; dx is held to the bound of one row's sums."""
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref
from tests.test_gpu_layers_norm import EPS, _forward

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# one of each way that a row is dealt out, with more rows than workgroups take at once; the last is too wide for registers
SHAPES = [(70_003, 32), (40_003, 100), (40_001, 130), (9_001, 256), (9_003, 512), (4_001, 1_000), (4_001, 2_047), (1_601, 4_096), (1_601, 8_192), (601, 9_001)]


def _whole(shape, most, g, t):
    return torch.randint(-most, most + 1, shape, generator=g).to(t)


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,d", SHAPES)
def test_sums_over_the_rows(n, d, t):
    g = torch.Generator().manual_seed(n + d)
    x, dy, gamma = _whole((n, d), 3, g, t), _whole((n, d), 2, g, t), _whole((d,), 2, g, t)
    mean, rstd = torch.zeros(n, device=DEV), torch.ones(n, device=DEV)
    xd, dyd = x.to(DEV), dy.to(DEV)
    assert 2 * 3 * n < 1 << 24
    dgamma, dbeta = (dy.double() * x.double()).sum(0).to(t), dy.double().sum(0).to(t)
    (dx, _, _), (off, _, _) = ref.layer_norm_backward(dy, x, mean, rstd, gamma)
    for source in (xd, B.grem_checkpoint_pack(xd)):
        got = B.grem_layer_norm_backward(dyd, source, mean, rstd, gamma.to(DEV))
        assert torch.equal(got[1].cpu(), dgamma) and torch.equal(got[2].cpu(), dbeta)
        ref.close(got[0], dx, off + ref.half_step(t) * (dx.abs() + off) + ref.least(t), "dx")


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,d", [(70_003, 32), (9_001, 1_000), (3_001, 8_192), (1_001, 9_001)])
def test_forward(n, d, t):
    g = torch.Generator().manual_seed(n + d)
    x = (torch.randn((n, d), generator=g) + torch.randn((n, 1), generator=g)).to(t)
    gamma, beta = (1 + 0.2 * torch.randn(d, generator=g)).to(t), torch.randn(d, generator=g).to(t)
    _forward(x.to(DEV), gamma, beta, EPS, f"{n} x {d}")
