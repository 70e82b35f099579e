"""A mean is the sum divided by the count: where the sums are exact the outputs are the quotients, rounded once, in every form that a
row is summed in.  (A sum times the rounded 1/41 is not 1 for 41 ones, and falls beside a tie of a 16-bit type for one in 150 sums of 7.)"""
import numpy as np
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _graph(n, most, seed, extra=()):
    rng = np.random.default_rng(seed)
    degrees = rng.integers(0, most + 1, n)
    degrees[:len(extra)] = extra
    rowptr = np.zeros(n + 1, np.int64)
    rowptr[1:] = np.cumsum(degrees)
    return rowptr, rng.integers(0, n, int(rowptr[-1])).astype(np.int32)


def _mean(rowptr, colidx, labels, x):
    n = len(rowptr) - 1
    out, _ = B.grem_neighbour_mean(torch.as_tensor(rowptr).to(DEV), torch.as_tensor(colidx).to(DEV), n, x.to(DEV),
                                   None if labels is None else torch.as_tensor(labels).to(DEV))
    return out.cpu()


# rows on the list, rows that are walked (many entries in all: rows are cut from 193 on, not from 129), rows in segments, more than 32 of them
@pytest.mark.parametrize("n,most,extra", [(2_000, 250, (41, 47, 83, 5_003)), (8_000, 300, (129, 191, 7_001))])
@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("d", [20, 100, 300])
def test_quotients(n, most, extra, t, d):
    rowptr, colidx = _graph(n, most, d + n, extra)
    x = torch.randint(-8, 9, (n, d), generator=torch.Generator().manual_seed(d)).to(t)
    for labels in (None, np.random.default_rng(n).integers(0, 2, n).astype(np.int32)):
        rows, cols = ref.kept_entries(rowptr, colidx, labels)
        sums = torch.zeros((n, d), dtype=torch.float64).index_add_(0, rows, x.double()[cols])
        counts = torch.bincount(rows, minlength=n).clamp(min=1).double().unsqueeze(1)
        # (the quotient in 64 bits, rounded to 32, is the quotient rounded to 32)
        assert torch.equal(_mean(rowptr, colidx, labels, x), (sums / counts).float().to(t))


@pytest.mark.parametrize("t", ref.TYPES)
def test_the_mean_of_equal_rows_is_the_row(t):
    degrees = [41, 47, 55, 61, 82, 83, 94, 97, 107, 109, 129, 500]
    rowptr = np.concatenate([[0], np.cumsum(degrees)]).astype(np.int64)
    x = torch.ones((len(degrees), 64), dtype=t)
    out = _mean(rowptr, np.arange(int(rowptr[-1]), dtype=np.int32) % len(degrees), None, x)
    assert torch.equal(out, x)


def test_sums_that_are_not_finite():
    rowptr, colidx = np.array([0, 3, 6, 9], np.int64), np.array([0, 1, 1, 1, 2, 1, 1, 1, 1], np.int32)
    x = torch.tensor([float("inf"), 1.0, float("nan")]).unsqueeze(1).repeat(1, 40)
    out = _mean(rowptr, colidx, None, x)
    assert torch.isinf(out[0]).all() and torch.isnan(out[1]).all() and torch.equal(out[2], torch.ones(40))
