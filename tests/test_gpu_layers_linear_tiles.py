"""The product over so many rows that a workgroup takes several tiles one after the other, the last of them cut off: the loads of the next
tile are under way while one is stored."""
import pytest
import torch

from paper_2502_17846_amd import binding as B
from tests import ref_layers as ref
from tests.test_gpu_layers_linear import ACTS, DEV, _backward, _data, _round

pytestmark = pytest.mark.gpu
# one for each size of tile; one step of the long axis and several, ends inside a step, a gradient's run that lies in both inputs
CASES = [(70_001, 64, 0, 256), (70_001, 72, 56, 256), (70_001, 200, 136, 264), (70_003, 40, 88, 128), (90_001, 24, 40, 64)]


@pytest.mark.parametrize("t", ref.TYPES)
@pytest.mark.parametrize("n,ka,kb,m", CASES)
def test_tile_after_tile(n, ka, kb, m, t):
    a, b, w, bias, residual, dout = _data(n, ka, kb, m, t)
    dev = [None if v is None else v.to(DEV) for v in (a, b, w, bias, residual)]
    for name, add, keep in (("gelu", True, True), ("none", False, False), ("relu", True, False), ("silu", False, True)):
        out = B.grem_linear(dev[0], dev[2], dev[3], dev[1], ACTS[name], dev[4] if add else None, want_pre=keep)
        want, z, tol, tol_z = ref.linear(a, b, w, bias, name, residual if add else None)
        if keep:
            out, pre = out
            ref.close(pre, z, _round(t, z, tol_z), f"{name} pre")
        ref.close(out, want, _round(t, want, tol), f"{name} out")
    _backward(dout, dev[0], dev[1], w, "silu", pre, a, b, "backward")


@pytest.mark.parametrize("t", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [1, 3, 5, 9, 63, 65, 100, 129])
def test_rows_that_end_inside_a_run(d, t):
    # both inputs and the outputs end there; NaN behind every row must not come in with the last run
    g = torch.Generator().manual_seed(d)
    wide = [torch.full((300, 160), float("nan"), dtype=t) for _ in range(4)]
    for v in wide:
        v[:, 2:2 + d] = torch.randn((300, d), generator=g).to(t)
    w = torch.full((d, 2 * d + 9), float("nan"), dtype=t)
    w[:, :2 * d] = (torch.randn((d, 2 * d), generator=g) / (2 * d) ** 0.5).to(t)
    a, b, dout, residual = (v[:, 2:2 + d] for v in wide)
    da, db, dd, dr = (v.to(DEV)[:, 2:2 + d] for v in wide)
    w, dw = w[:, :2 * d], w.to(DEV)[:, :2 * d]
    out, pre = B.grem_linear(da, dw, None, db, B.ACT_SILU, dr, want_pre=True)
    want, z, tol, tol_z = ref.linear(a, b, w, None, "silu", residual)
    ref.close(out, want, _round(t, want, tol), "out")
    for source in ((da, db), (B.grem_checkpoint_pack(da), B.grem_checkpoint_pack(db))):
        values = (a, b) if source[0] is da else tuple(ref.pack(v)[2].to(t) for v in (a, b))
        for name in ("silu", "none"):
            got = B.grem_linear_backward(dd, source[0], dw, source[1], ACTS[name], pre if name == "silu" else None)
            wants, tols = ref.linear_backward(dout, *values, w, name, pre)
            for part, g_, v, e in zip(("da", "db", "dw", "dbias"), got, wants, tols):
                ref.close(g_, v, _round(t, v, e), f"{name} {part}")
