"""The product with bias, activation and residual, and its backward pass, against the formulas in 64 bits."""
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ACTS = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "gelu": B.ACT_GELU, "silu": B.ACT_SILU}
# (n, ka, kb, m)
SHAPES = [(1, 1, 0, 1), (1, 256, 256, 256), (3, 5, 7, 9), (16, 64, 0, 64), (17, 65, 1, 33), (40, 100, 100, 47), (64, 512, 0, 16), (65, 8, 8, 130),
          (129, 40, 24, 257), (300, 128, 128, 128), (255, 72, 0, 520), (1000, 33, 95, 100), (513, 520, 264, 264)]


def _data(n, ka, kb, m, t, seed=0):
    g = torch.Generator().manual_seed(seed + n + 3 * ka + 5 * kb + 7 * m)
    a = torch.randn((n, ka), generator=g).to(t)
    b = torch.randn((n, kb), generator=g).to(t) if kb else None
    w = (torch.randn((m, ka + kb), generator=g) / (ka + kb) ** 0.5).to(t)
    bias, residual, dout = torch.randn(m, generator=g).to(t), torch.randn((n, m), generator=g).to(t), torch.randn((n, m), generator=g).to(t)
    return a, b, w, bias, residual, dout


def _dev(v):
    return None if v is None else v.to(DEV)


def _round(t, want, tol):
    return tol + ref.half_step(t) * (want.abs() + tol) + ref.least(t)


def _forward(a, b, w, bias, name, residual, what):
    t = w.dtype
    out, pre = B.grem_linear(_dev(a), _dev(w), _dev(bias), _dev(b), ACTS[name], _dev(residual), want_pre=True)
    want, z, tol, tol_z = ref.linear(a, b, w, bias, name, residual)
    ref.close(pre, z, _round(t, z, tol_z), what + " pre")
    ref.close(out, want, _round(t, want, tol), what + " out")
    return pre


def _backward(dout, a, b, w, name, pre, va, vb, what):
    t = w.dtype
    got = B.grem_linear_backward(_dev(dout), a, _dev(w), b, ACTS[name], pre)
    want, tol = ref.linear_backward(dout, va, vb, w, name, pre)
    for part, g, v, e in zip(("da", "db", "dw", "dbias"), got, want, tol):
        if v is None:
            assert g is None
        else:
            ref.close(g, v, _round(t, v, e), f"{what} {part}")


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,ka,kb,m", SHAPES)
def test_both_passes(n, ka, kb, m, t):
    a, b, w, bias, residual, dout = _data(n, ka, kb, m, t)
    names = list(ACTS)
    name = names[(n + ka + m) % 4]
    what = f"{n}, {ka}+{kb} to {m}, {name}"
    pre = _forward(a, b, w, bias, name, residual if n % 2 else None, what)
    _backward(dout, _dev(a), _dev(b), w, name, pre, a, b, what)
    packed = [None if v is None else B.grem_checkpoint_pack(_dev(v)) for v in (a, b)]
    values = [None if v is None else ref.pack(v)[2].to(t) for v in (a, b)]
    _backward(dout, packed[0], packed[1], w, name, pre, values[0], values[1], what + " from 8 bits")


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("name", list(ACTS))
def test_activations_over_their_range(name, t):
    # one input column, weight 1: z runs over the whole range of the activation, both tails included
    z = torch.cat([torch.linspace(-20, 20, 2001), torch.tensor([0.0, -0.0, 100.0, -100.0, 1e4, -1e4])]).to(t).unsqueeze(1)
    w = torch.ones((1, 1), dtype=t)
    pre = _forward(z, None, w, None, name, None, name)
    dout = torch.ones_like(z)
    _backward(dout, _dev(z), None, w, name, pre, z, None, name)


@pytest.mark.parametrize("t", ref.TYPES)
def test_strides_and_odd_bases(t):
    g = torch.Generator().manual_seed(4)
    wide = torch.randn((200, 210), generator=g).to(t)
    dev = wide.to(DEV)
    a, b, w, dout = wide[::2, 1:68], wide[1::2, 5:38], wide[:31, 3:103], wide[::2, 70:101]
    da, db, dw, dd = dev[::2, 1:68], dev[1::2, 5:38], dev[:31, 3:103], dev[::2, 70:101]
    out, pre = B.grem_linear(da, dw, None, db, B.ACT_SILU, dev[1::2, 101:132], want_pre=True)
    want, z, tol, tol_z = ref.linear(a, b, w, None, "silu", wide[1::2, 101:132])
    ref.close(out, want, _round(t, want, tol), "strided out")
    got = B.grem_linear_backward(dd, da, dw, db, B.ACT_SILU, pre)
    want, tol = ref.linear_backward(dout, a, b, w, "silu", pre)
    for g_, v, e in zip(got, want, tol):
        ref.close(g_, v, _round(t, v, e), "strided gradient")


def test_values_beyond_a_row_are_not_multiplied():
    # NaN right after every row and after a's part of the weights' rows stays out of the sums
    t = torch.bfloat16
    wide = torch.full((40, 64), float("nan"), dtype=t, device=DEV)
    wide[:, :21] = 1.0
    w = torch.full((9, 64), float("nan"), dtype=t, device=DEV)
    w[:, :21] = 2.0
    out = B.grem_linear(wide[:, :21], w[:, :21])
    assert torch.equal(out, torch.full_like(out, 42.0))
    da, _, dw, dbias = B.grem_linear_backward(out, wide[:, :21], w[:, :21])
    assert torch.isfinite(da).all() and torch.isfinite(dw).all() and torch.isfinite(dbias).all()


def test_a_bad_row_stays_alone():
    a = torch.ones((70, 30), device=DEV)
    a[33, 4] = float("nan")
    out = B.grem_linear(a, torch.ones((20, 30), device=DEV), act=B.ACT_RELU)
    assert torch.isnan(out).any(1).cpu().tolist() == [r == 33 for r in range(70)] and torch.isnan(out[33]).all()


def test_residual_in_place_and_parts_that_are_not_wanted():
    a, b, w, bias, residual, dout = _data(90, 40, 24, 50, torch.float16)
    want = B.grem_linear(_dev(a), _dev(w), _dev(bias), _dev(b), B.ACT_GELU, _dev(residual))
    r = _dev(residual)
    B.grem_linear(_dev(a), _dev(w), _dev(bias), _dev(b), B.ACT_GELU, r, out=r)
    assert torch.equal(r, want)
    full = B.grem_linear_backward(_dev(dout), _dev(a), _dev(w), _dev(b))
    inputs = B.grem_linear_backward(_dev(dout), _dev(a), _dev(w), _dev(b), want_params=False)
    params = B.grem_linear_backward(_dev(dout), _dev(a), _dev(w), _dev(b), want_inputs=False)
    assert torch.equal(inputs[0], full[0]) and torch.equal(inputs[1], full[1]) and inputs[2] is None and inputs[3] is None
    assert torch.equal(params[2], full[2]) and torch.equal(params[3], full[3]) and params[0] is None and params[1] is None


def test_no_rows():
    w = torch.ones((6, 10), device=DEV)
    e = torch.empty((0, 10), device=DEV)
    assert B.grem_linear(e, w).shape == (0, 6)
    da, db, dw, dbias = B.grem_linear_backward(torch.empty((0, 6), device=DEV), e, w)
    assert da.shape == (0, 10) and dw.abs().sum() == 0 and dbias.abs().sum() == 0


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_many_rows(t):
    # rows enough for the weights' gradient to be summed in stretches, the last of them short
    n, ka, kb, m = 20_011, 72, 40, 136
    a, b, w, bias, residual, dout = _data(n, ka, kb, m, t)
    pre = _forward(a, b, w, bias, "gelu", residual, "many")
    _backward(dout, _dev(a), _dev(b), w, "gelu", pre, a, b, "many")


def test_gradient_against_differences():
    g = torch.Generator().manual_seed(6)
    n, ka, m = 3, 5, 4
    a, w, dout = torch.randn((n, ka), generator=g, dtype=torch.float64), torch.randn((m, ka), generator=g, dtype=torch.float64), torch.randn((n, m), generator=g, dtype=torch.float64)
    for name in ("gelu", "silu"):
        def f(x, y):
            return float((ref.act(x @ y.T, name) * dout).sum())

        h = 1e-5
        diff_a, diff_w = torch.zeros_like(a), torch.zeros_like(w)
        for v, diff, left in ((a, diff_a, True), (w, diff_w, False)):
            for i in range(v.shape[0]):
                for j in range(v.shape[1]):
                    e = torch.zeros_like(v)
                    e[i, j] = h
                    diff[i, j] = (f(a + e, w) - f(a - e, w) if left else f(a, w + e) - f(a, w - e)) / (2 * h)
        af, wf, df = (v.float().to(DEV) for v in (a, w, dout))
        _, pre = B.grem_linear(af, wf, act=ACTS[name], want_pre=True)
        da, _, dw, _ = B.grem_linear_backward(df, af, wf, act=ACTS[name], pre=pre)
        assert (da.cpu().double() - diff_a).abs().max() < 1e-5 * max(1.0, diff_a.abs().max())
        assert (dw.cpu().double() - diff_w).abs().max() < 1e-5 * max(1.0, diff_w.abs().max())
