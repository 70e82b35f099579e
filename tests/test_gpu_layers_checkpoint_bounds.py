"""How far an 8-bit checkpoint's values are from what was packed, as include/grem.h states it, over the whole range of each type; and the
codes, exponents and values of many rows, of which a workgroup takes several."""
import numpy as np
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref
from tests.ref_pack import pack

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("t", ref.TYPES)
def test_distance(t):
    g = torch.Generator().manual_seed(3)
    f = torch.finfo(t)
    # groups whose largest values run through every binade of the type, the last one's in steps up to its largest number
    exponents = torch.arange(-24 if t == torch.float16 else -133, 16 if t == torch.float16 else 128)
    size = torch.cat([torch.exp2(exponents.double()), torch.linspace(0.5, 1, 200, dtype=torch.float64) * f.max])
    x = torch.rand((len(size), 32), generator=g, dtype=torch.float64) * 2 - 1
    x[:, 5] = torch.where(torch.arange(len(size)) % 2 == 0, 1.0, -1.0)
    x = (x * size.unsqueeze(1)).to(t)
    assert torch.isfinite(x).all()
    kept = B.grem_checkpoint_pack(x.to(DEV))
    back = B.grem_checkpoint_unpack(kept).cpu()
    assert torch.isfinite(back).all()
    e = kept.exponents.cpu().double() - 130
    largest = x.double().abs().amax(1, keepdim=True)
    top = 10 if t == torch.float16 else 122
    stopped = (e == top) & (x.double().abs() >= 63.5 * torch.exp2(e))
    off = (x.double() - back.double()).abs()
    # (below half precision's normal range a value read back is rounded once more)
    assert (off <= torch.where(stopped, torch.exp2(e), torch.exp2(e - 1)) + ref.least(t)).all()
    assert stopped.any() and (kept.codes.cpu()[stopped].abs() == 63).all() and (off[stopped] > torch.exp2(e - 1).expand_as(off)[stopped]).any()
    normal = (e > -130).squeeze(1)
    assert (torch.exp2(e - 1) <= largest / 127)[normal].all() and (torch.exp2(e - 1) >= largest / 254)[normal].all()


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,d", [(9_001, 31), (9_001, 100), (70_003, 100), (70_003, 31), (20_011, 256)])
def test_many_rows(n, d, t):
    g = torch.Generator().manual_seed(n + d)
    x = torch.randn((n, d), generator=g) * torch.exp2(torch.randint(-12, 12, (n, -(-d // 32)), generator=g).float()).repeat_interleave(32, 1)[:, :d]
    x[n // 2, d - 1], x[n - 1, 0], x[n - 2, d // 2] = float("nan"), float("inf"), 0.0
    x = x.to(t)
    codes, exponents, values = pack(x)
    kept = B.grem_checkpoint_pack(x.to(DEV))
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.exponents.cpu(), exponents)
    back = B.grem_checkpoint_unpack(kept).cpu()
    want = values.to(t)
    assert torch.equal(torch.isnan(back), torch.isnan(want)) and torch.equal(torch.nan_to_num(back), torch.nan_to_num(want))
