"""Layer norm and its backward pass against the formulas in 64 bits."""
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5
# one lane to a whole workgroup a row, in and out of the widths that fit registers
SHAPES = [(1, 1), (3, 2), (1, 17), (5, 64), (33, 100), (9, 128), (1025, 130), (70, 256), (13, 511), (8, 1000), (300, 1024), (6, 2047),
          (5, 2048), (4, 4099), (3, 8192), (3, 9001)]


def _data(n, d, t, seed=0):
    g = torch.Generator().manual_seed(seed + 7 * n + d)
    x = (torch.randn((n, d), generator=g) * (torch.rand(d, generator=g) + 0.5) + torch.randn(d, generator=g)).to(t)
    gamma, beta = (1 + 0.2 * torch.randn(d, generator=g)).to(t), torch.randn(d, generator=g).to(t)
    return x, gamma, beta, torch.randn((n, d), generator=g).to(t)


def _forward(x_dev, gamma, beta, eps, what):
    t = x_dev.dtype
    y, mean, rstd = B.grem_layer_norm(x_dev, None if gamma is None else gamma.to(DEV), None if beta is None else beta.to(DEV), eps)
    want, tol = ref.layer_norm(x_dev, gamma, beta, eps)
    ref.close(y, want[0], tol[0] + ref.half_step(t) * (want[0].abs() + tol[0]) + ref.least(t), what + " y")
    ref.close(mean, want[1], tol[1], what + " mean")
    ref.close(rstd, want[2], tol[2], what + " rstd")
    return mean, rstd


def _backward(dy, source, x, mean, rstd, gamma, what):
    t = dy.dtype
    got = B.grem_layer_norm_backward(dy, source, mean, rstd, None if gamma is None else gamma.to(DEV))
    want, tol = ref.layer_norm_backward(dy, x, mean, rstd, gamma)
    for name, g, w, e in zip(("dx", "dgamma", "dbeta"), got, want, tol):
        ref.close(g, w, e + ref.half_step(t) * (w.abs() + e) + ref.least(t), f"{what} {name}")
    return got


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,d", SHAPES)
def test_both_passes(n, d, t):
    x, gamma, beta, dy = _data(n, d, t)
    xd, dyd = x.to(DEV), dy.to(DEV)
    mean, rstd = _forward(xd, gamma, beta, EPS, f"{n} x {d}")
    _backward(dyd, xd, x, mean, rstd, gamma, f"{n} x {d}")
    ck = B.grem_checkpoint_pack(xd)
    _backward(dyd, ck, ref.pack(x)[2], mean, rstd, gamma, f"{n} x {d} from 8 bits")


@pytest.mark.parametrize("t", ref.TYPES)
def test_strides_odd_bases_and_no_parameters(t):
    x, _, _, dy = _data(41, 300, t, 3)
    xd, dyd = x.to(DEV), dy.to(DEV)
    for lo, hi in ((1, 258), (3, 131), (2, 3)):
        a, b = xd[::2, lo:hi], dyd[::2, lo:hi]
        mean, rstd = _forward(a, None, None, 1e-3, f"[{lo}:{hi}]")
        _backward(b, a, x[::2, lo:hi], mean, rstd, None, f"[{lo}:{hi}]")


def test_constant_rows_and_a_large_mean():
    x = torch.full((3, 96), 7.0)
    x[1] = 0.0
    x[2] = 1.0e4 + torch.arange(96) * 0.25             # digits of the variance must not cancel
    mean, rstd = _forward(x.to(DEV), None, None, EPS, "constant")
    dy = torch.ones((3, 96)) * torch.arange(96)
    _backward(dy.to(DEV), x.to(DEV), x, mean, rstd, None, "constant")


def test_a_bad_row_stays_alone():
    x, gamma, beta, dy = _data(9, 200, torch.float32, 5)
    x[4, 7], x[6, 0] = float("nan"), float("inf")
    y, mean, rstd = B.grem_layer_norm(x.to(DEV), gamma.to(DEV), beta.to(DEV))
    bad = torch.isnan(y).any(1).cpu()
    assert bad.tolist() == [r in (4, 6) for r in range(9)] and torch.isnan(y[4]).all() and torch.isnan(y[6]).all()
    dx, _, _ = B.grem_layer_norm_backward(dy.to(DEV), x.to(DEV), mean, rstd, gamma.to(DEV))
    assert torch.isnan(dx).any(1).cpu().tolist() == [r in (4, 6) for r in range(9)]


def test_no_rows():
    e = torch.empty((0, 24), device=DEV)
    y, mean, rstd = B.grem_layer_norm(e)
    assert y.shape == (0, 24) and mean.numel() == 0
    dx, dg, db = B.grem_layer_norm_backward(e, e, mean, rstd)
    assert dx.shape == (0, 24) and dg.cpu().tolist() == [0.0] * 24 and db.cpu().tolist() == [0.0] * 24


def test_gradient_against_differences():
    n, d = 4, 10
    g = torch.Generator().manual_seed(2)
    x, dy = torch.randn((n, d), generator=g, dtype=torch.float64), torch.randn((n, d), generator=g, dtype=torch.float64)
    gamma = torch.rand(d, generator=g, dtype=torch.float64) + 0.5

    def f(v):
        return float((ref.layer_norm(v, gamma, None, EPS)[0][0] * dy).sum())

    h, diff = 1e-5, torch.zeros_like(x)
    for i in range(n):
        for j in range(d):
            e = torch.zeros_like(x)
            e[i, j] = h
            diff[i, j] = (f(x + e) - f(x - e)) / (2 * h)
    xf, dyf, gf = (v.float().to(DEV) for v in (x, dy, gamma))
    _, mean, rstd = B.grem_layer_norm(xf, gf)
    dx, _, _ = B.grem_layer_norm_backward(dyf, xf, mean, rstd, gf)
    assert (dx.cpu().double() - diff).abs().max() < 1e-4 * diff.abs().max()      # 32-bit inputs: 2^-24 * a few dozen; h^2: 1e-10
