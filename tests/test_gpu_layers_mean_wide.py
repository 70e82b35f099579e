"""The neighbour mean of rows so wide that several waves share a segment's columns."""
import numpy as np
import pytest
import torch

from tests.test_gpu_layers_mean import _check, _random, _values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [16_400, 33_001, 50_000])
def test_long_rows(d, t):
    rowptr, colidx = _random(12, 10, d, np.int64, [(2, 129), (5, 700), (11, 400)])
    labels = np.random.default_rng(d).integers(0, 2, 12).astype(np.int32)
    for given in (None, labels):
        _check(rowptr, colidx, given, _values(12, d, t, 1), _values(12, d, t, 2), f"d={d}")
