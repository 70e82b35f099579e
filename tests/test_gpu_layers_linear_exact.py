"""The product's backward pass over many rows, on whole numbers: every sum is a whole number below 2^24, exact in 32 bits in whatever order,
so that gradients are the formula's, rounded once, and a row that is lost or taken twice is seen.  From values and from 8 bits (whole
numbers up to 3 are kept exactly), with both tiles of the weights' gradient."""
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# (n, ka, kb, m): whole tiles of 128 and of 256, rows that end inside a run, one input and two, a last stretch of a few rows
SHAPES = [(4_096, 256, 256, 256), (4_611, 264, 136, 264), (4_611, 257, 129, 257), (20_011, 264, 136, 257), (20_011, 257, 0, 264), (65_793, 136, 40, 136),
          (70_001, 200, 136, 264), (70_001, 129, 131, 130), (90_001, 64, 0, 64), (8_193, 520, 8, 132)]


def _whole(shape, most, g, t):
    return torch.randint(-most, most + 1, shape, generator=g).to(t)


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,ka,kb,m", SHAPES)
def test_gradients(n, ka, kb, m, t):
    g = torch.Generator().manual_seed(n + ka + kb + m)
    a, b = _whole((n, ka), 3, g, t), _whole((n, kb), 3, g, t) if kb else None
    w, dout, pre = _whole((m, ka + kb), 3, g, t), _whole((n, m), 2, g, t), _whole((n, m), 1, g, t)
    dev = [None if v is None else v.to(DEV) for v in (a, b)]
    packed = [None if v is None else B.grem_checkpoint_pack(v) for v in dev]
    for v, p in zip(dev, packed):
        assert v is None or torch.equal(B.grem_checkpoint_unpack(p), v)
    x = (a if b is None else torch.cat([a, b], 1)).double()
    for name, dz in ((B.ACT_NONE, dout), (B.ACT_RELU, torch.where(pre > 0, dout, torch.zeros_like(dout)))):
        dz = dz.double()
        assert 2 * 3 * n < 1 << 24 and 2 * 3 * m < 1 << 24
        back, want = dz @ w.double(), ((dz.T @ x).to(t), dz.sum(0).to(t))
        for sources in (dev, packed):
            da, db, dw, dbias = B.grem_linear_backward(dout.to(DEV), sources[0], w.to(DEV), sources[1], name, None if name == B.ACT_NONE else pre.to(DEV))
            assert torch.equal(dw.cpu(), want[0]) and torch.equal(dbias.cpu(), want[1])
            assert torch.equal(da.cpu(), back[:, :ka].to(t)) and (db is None or torch.equal(db.cpu(), back[:, ka:].to(t)))
