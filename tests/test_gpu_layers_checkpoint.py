"""8-bit checkpoints against the rule itself: codes and exponent bytes equal, values exact."""
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rows(n, d, t, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, d), generator=g) * torch.exp2(torch.randint(-20, 12, (n, -(-d // 32)), generator=g).float()).repeat_interleave(32, 1)[:, :d]
    return x.to(t)


def _check(x_dev, x):
    codes, exponents, values = ref.pack(x)
    ck = B.grem_checkpoint_pack(x_dev)
    assert torch.equal(ck.codes.cpu(), codes) and torch.equal(ck.exponents.cpu(), exponents)
    back = B.grem_checkpoint_unpack(ck)
    assert back.dtype == x.dtype
    want = values.to(x.dtype)
    assert torch.equal(torch.isnan(back.cpu()), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(back.cpu()), torch.nan_to_num(want))


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,d", [(1, 1), (1, 31), (3, 32), (5, 33), (17, 100), (257, 64), (64, 255), (3, 1056), (1, 40_000)])
def test_codes_and_values(n, d, t):
    x = _rows(n, d, t, n * 1000 + d)
    _check(x.to(DEV), x)


@pytest.mark.parametrize("t", ref.TYPES)
def test_strided_rows_at_odd_places(t):
    wide = _rows(50, 150, t, 1)
    dev = wide.to(DEV)
    for lo, hi in ((0, 96), (1, 98), (3, 40), (7, 150)):
        _check(dev[::2, lo:hi], wide[::2, lo:hi])


@pytest.mark.parametrize("t", ref.TYPES)
def test_the_ends_of_the_range(t):
    f = torch.finfo(t)
    x = torch.zeros((12, 32), dtype=t)
    x[0, 3] = f.max
    x[1, 3], x[1, 4] = f.min, f.max / 2
    x[2, :] = f.tiny
    x[3, 0] = torch.finfo(t).smallest_normal * f.eps          # the smallest number
    x[4, 5] = float("nan")
    x[5, 6], x[5, 7] = float("inf"), 1.0
    x[6, 8] = float("-inf")
    x[7, :] = torch.arange(32).to(t) * 4                      # 124: codes are the numbers themselves
    x[8, 0], x[8, 1], x[8, 2], x[8, 3] = 127.0, 0.5, 1.5, -2.5     # ties go to even
    x[9, 0], x[9, 1] = 128.0, 3.0
    x[10, 0] = 127.5 if t != torch.bfloat16 else 254.0
    x[11, 0] = -1.0
    _check(x.to(DEV), x)


def test_nothing():
    ck = B.grem_checkpoint_pack(torch.empty((0, 5), device=DEV))
    assert ck.codes.shape == (0, 5) and B.grem_checkpoint_unpack(ck).shape == (0, 5)
