"""The two statements of the checkpoints' rule that the tests use agree."""
import pytest
import torch

from tests import ref_layers as ref
from tests.ref_pack import pack


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,d", [(60, 1), (40, 31), (40, 100), (7, 256)])
def test_both_forms(n, d, t):
    g = torch.Generator().manual_seed(n * d)
    f = torch.finfo(t)
    x = torch.randn((n, d), generator=g) * torch.exp2(torch.randint(-14, 13, (n, 1), generator=g).float())
    x[0], x[1] = 0.0, 127.0
    x = x.to(t)
    x[2, 0], x[3, d - 1], x[4, 0], x[5, d // 2] = f.max, f.tiny * f.eps, float("nan"), float("-inf")
    for got, want in zip(pack(x), ref.pack(x)):
        assert got.dtype == want.dtype and torch.equal(torch.nan_to_num(got.double(), nan=0.5), torch.nan_to_num(want.double(), nan=0.5))
