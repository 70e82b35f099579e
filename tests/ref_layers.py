"""The layer operators' definitions in 64 bits (torch on the CPU), with a bound for what 32-bit sums and the roundings to a type may add.

half_step(t) is the largest relative error of one rounding to nearest.  A sum of K terms in 32 bits, in any order, is off by
at most K * 2^-24 of the sum of the terms' sizes (to first order); SLACK more steps stand for the operations around it."""
import numpy as np
import torch

F32 = 2.0 ** -24
SLACK = 16
TYPES = [torch.float32, torch.bfloat16, torch.float16]
GROUP = 32


def half_step(t):
    return torch.finfo(t).eps / 2


def least(t):
    """Half a step of the type's smallest numbers."""
    return 2.0 ** -150 if t == torch.float32 else 2.0 ** -134 if t == torch.bfloat16 else 2.0 ** -25


def close(got, want, tol, what):
    """|got - want| <= tol everywhere, NaN and infinities in the same places."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), f"{what}: finite in other places"
    assert torch.equal(torch.isnan(want), torch.isnan(got)), f"{what}: NaN in other places"
    off = ((got - want).abs() - tol)[fine]
    assert off.numel() == 0 or off.max() <= 0, f"{what}: {int((off > 0).sum())} of {off.numel()} values off, by up to {float(off.max())} more than allowed"


# ---- mean over the neighbours of the same partition -------------------------------------------------------------------

def kept_entries(rowptr, colidx, labels):
    rowptr, colidx = np.asarray(rowptr, np.int64), np.asarray(colidx, np.int64)
    rows = np.repeat(np.arange(len(rowptr) - 1), np.diff(rowptr))
    keep = np.ones(len(rows), bool) if labels is None else (labels[rows] == labels[colidx]) & (labels[rows] >= 0)
    return torch.as_tensor(rows[keep]), torch.as_tensor(colidx[keep])


def neighbour_mean(rowptr, colidx, labels, x):
    """(out, counts, bound without the rounding)"""
    rows, cols = kept_entries(rowptr, colidx, labels)
    n = x.shape[0]
    counts = torch.bincount(rows, minlength=n)
    c = counts.clamp(min=1).double().unsqueeze(1)
    zero = torch.zeros(x.shape, dtype=torch.float64)
    xd = x.cpu().double()
    out = zero.clone().index_add_(0, rows, xd[cols]) / c
    size = zero.clone().index_add_(0, rows, xd[cols].abs()) / c
    return out, counts.int(), (counts.unsqueeze(1) + SLACK) * F32 * size


def neighbour_mean_backward(rowptr, colidx, labels, dout, counts):
    """dx of the forward graph (rowptr, colidx), entry by entry."""
    rows, cols = kept_entries(rowptr, colidx, labels)
    g = dout.cpu().double() / counts.clamp(min=1).double().unsqueeze(1)
    zero = torch.zeros(dout.shape, dtype=torch.float64)
    dx = zero.clone().index_add_(0, cols, g[rows])
    size = zero.clone().index_add_(0, cols, g[rows].abs())
    used = torch.bincount(cols, minlength=dout.shape[0])
    return dx, (used.unsqueeze(1) + SLACK) * F32 * size


# ---- the product ----------------------------------------------------------------------------------------------------------

def act(z, name):
    if name == "relu":
        return torch.where(torch.isnan(z), z, z.clamp(min=0))
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / 2 ** 0.5)
    return z * torch.sigmoid(z) if name == "silu" else z


def slope(z, name):
    if name == "relu":
        return torch.where(torch.isnan(z), z, (z > 0).double())
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / 2 ** 0.5) + z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    s = torch.sigmoid(z)
    return s + z * s * (1 - s) if name == "silu" else torch.ones_like(z)


def linear(a, b, w, bias, name, residual):
    """(out, z, bounds of both without the rounding); no slope of an activation is above 1.13."""
    x = a.cpu().double() if b is None else torch.cat([a.cpu().double(), b.cpu().double()], 1)
    wd = w.cpu().double()
    z, size = x @ wd.T, x.abs() @ wd.abs().T
    if bias is not None:
        z, size = z + bias.cpu().double(), size + bias.cpu().double().abs()
    tol = (x.shape[1] + SLACK) * F32 * size
    out, tol_out = act(z, name), 1.13 * tol + SLACK * F32 * z.abs()
    if residual is not None:
        out = out + residual.cpu().double()
        tol_out = tol_out + F32 * (out.abs() + residual.cpu().double().abs())
    return out, z, tol_out, tol


def linear_backward(dout, a, b, w, name, pre):
    """((da, db, dw, dbias), their bounds without the last rounding): dz is rounded to the type before the products."""
    t = dout.dtype
    x = a.double() if b is None else torch.cat([a.double(), b.double()], 1)
    dz, wd, n, m = dout.cpu().double(), w.cpu().double(), dout.shape[0], dout.shape[1]
    own = torch.zeros_like(dz)
    if name != "none":
        z = pre.cpu().double()
        s = slope(z, name)
        # the slope's own error in 32 bits, a few steps of its terms, and dz's rounding
        own = SLACK * F32 * dz.abs() * (1 + z.abs())
        dz = dz * s
    rounded = own + (half_step(t) * dz.abs() + least(t) if name != "none" else 0)
    back, tol_back = dz @ wd, ((m + SLACK) * F32 * dz.abs() + rounded) @ wd.abs()
    dw, tol_w = dz.T @ x, ((n + SLACK) * F32 * dz.abs() + rounded).T @ x.abs()
    dbias, tol_bias = dz.sum(0), ((n + SLACK) * F32 * dz.abs() + own).sum(0)
    ka = a.shape[1]
    return (back[:, :ka], None if b is None else back[:, ka:], dw, dbias), (tol_back[:, :ka], None if b is None else tol_back[:, ka:], tol_w, tol_bias)


# ---- layer norm ------------------------------------------------------------------------------------------------------------

def layer_norm(x, gamma, beta, eps):
    """((y, mean, rstd), bounds without y's rounding)"""
    x = x.cpu().double()
    d = x.shape[1]
    mean = x.mean(1, keepdim=True)
    tol_mean = (d + SLACK) * F32 * x.abs().mean(1, keepdim=True)
    var = ((x - mean) ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    # the variance about a mean that is off by e is off by e^2, and by the sums' and the differences' roundings
    off_var = tol_mean ** 2 + (d + SLACK) * F32 * var + 2 * F32 * (x.abs() * (x - mean).abs()).mean(1, keepdim=True)
    rel = 0.5 * off_var * rstd ** 2 + SLACK * F32
    hat = (x - mean) * rstd
    tol_hat = hat.abs() * rel + (tol_mean + F32 * x.abs()) * rstd * (1 + rel)
    g = torch.ones(d, dtype=torch.float64) if gamma is None else gamma.cpu().double()
    b = torch.zeros(d, dtype=torch.float64) if beta is None else beta.cpu().double()
    y = hat * g + b
    return (y, mean[:, 0], rstd[:, 0]), (tol_hat * g.abs() + 4 * F32 * (y.abs() + b.abs()), tol_mean[:, 0], (rel * rstd)[:, 0])


def layer_norm_backward(dy, x, mean, rstd, gamma):
    """((dx, dgamma, dbeta), bounds without the rounding); mean and rstd as they are given."""
    dy, x, mu, rs = dy.cpu().double(), x.cpu().double(), mean.cpu().double().unsqueeze(1), rstd.cpu().double().unsqueeze(1)
    n, d = dy.shape
    g = torch.ones(d, dtype=torch.float64) if gamma is None else gamma.cpu().double()
    hat = (x - mu) * rs
    tol_hat = 4 * F32 * (x.abs() + mu.abs()) * rs
    t = dy * g
    s1, s2 = t.mean(1, keepdim=True), (t * hat).mean(1, keepdim=True)
    k = (d + SLACK) * F32
    tol_s2 = k * (t * hat).abs().mean(1, keepdim=True) + (t.abs() * tol_hat).mean(1, keepdim=True)
    dx = rs * (t - s1 - hat * s2)
    tol = rs * (SLACK * F32 * (t.abs() + s1.abs() + (hat * s2).abs()) + k * t.abs().mean(1, keepdim=True) + tol_hat * s2.abs() + hat.abs() * tol_s2)
    dg, db = (dy * hat).sum(0), dy.sum(0)
    tol_dg = (n + SLACK) * F32 * (dy * hat).abs().sum(0) + (dy.abs() * tol_hat).sum(0)
    return (dx, dg, db), (tol, tol_dg, (n + SLACK) * F32 * dy.abs().sum(0))


# ---- checkpoints ------------------------------------------------------------------------------------------------------------

def pack(x):
    """(codes, exponent bytes, values) by the rule itself, value by value in 64 bits."""
    top = 10 if x.dtype == torch.float16 else 122
    xd = x.detach().cpu().double().numpy()
    n, d = xd.shape
    groups = -(-d // GROUP)
    codes, bytes_, values = np.zeros((n, d), np.int8), np.zeros((n, groups), np.uint8), np.zeros((n, d))
    for r in range(n):
        for g in range(groups):
            v = xd[r, g * GROUP:(g + 1) * GROUP]
            at = slice(g * GROUP, g * GROUP + len(v))
            if not np.all(np.isfinite(v)):
                bytes_[r, g], values[r, at] = 255, np.nan
                continue
            largest = np.abs(v).max()
            e = -130
            while largest > 127 * 2.0 ** e:
                e += 1
            q = np.rint(v / 2.0 ** e)
            if e == top:
                q = np.clip(q, -63, 63)
            codes[r, at], bytes_[r, g], values[r, at] = q, e + 130, q * 2.0 ** e
    return torch.as_tensor(codes), torch.as_tensor(bytes_), torch.as_tensor(values)
