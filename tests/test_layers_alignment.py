"""Pointers that the layer operators refuse for their alignment, at the C entry points: checks come before any launch, the pointers are
never followed."""
import os

import pytest

from paper_2502_17846_amd import binding as B
from tests.test_layers_refusals import BF16, F16, F32, P, _call, _expect, _rows


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2502_17846_amd import build
        build.build_library()
    return B.load()


def test_neighbour_mean(lib):
    need = lib.grem_neighbour_mean_bytes(F32, 10, 100_000, 64, 1)
    args = dict(rowptr=P, bits=64, colidx=P, nnz=100_000, n=10, labels=P, type=F32, d=64, x=P, ldx=64, out=P, ldo=64, counts=P, ws=P, bytes=need,
                stream=None)
    bad = [dict(rowptr=P + 4), dict(bits=32, rowptr=P + 2), dict(colidx=P + 2), dict(labels=P + 1), dict(counts=P + 2), dict(ws=P + 128), dict(ws=P + 4)]
    _expect(lib.grem_neighbour_mean, "rowptr bits colidx nnz n labels type d x ldx out ldo counts ws bytes stream", args, bad)
    _expect(lib.grem_neighbour_mean_backward, "rowptr bits colidx nnz n labels counts type d x ldx out ldo ws bytes stream", args, bad)


def test_linear_backward(lib):
    order = "type n m dout ldd act pre ldp a ka b kb w ldw da ldda db lddb dw lddw dbias ws bytes stream"
    need = lib.grem_linear_backward_bytes(F16, 10, 32, 64, 16, 3)
    args = dict(type=F16, n=10, m=32, dout=P, ldd=32, act=3, pre=P, ldp=32, a=_rows(), ka=64, b=_rows(stride=16), kb=16, w=P, ldw=80, da=P, ldda=64,
                db=P, lddb=16, dw=P, lddw=80, dbias=P, ws=P, bytes=need, stream=None)
    _expect(lib.grem_linear_backward, order, args, [dict(ws=P + 16), dict(ws=P + 128)])


def test_layer_norm(lib):
    args = dict(type=BF16, n=10, d=64, x=P, ldx=64, gamma=P, beta=P, eps=1e-5, y=P, ldy=64, mean=P, rstd=P, stream=None)
    _expect(lib.grem_layer_norm, "type n d x ldx gamma beta eps y ldy mean rstd stream", args, [dict(mean=P + 2), dict(rstd=P + 1)])
    need = lib.grem_layer_norm_backward_bytes(10, 64)
    args = dict(type=BF16, n=10, d=64, dy=P, lddy=64, x=_rows(), mean=P, rstd=P, gamma=P, dx=P, lddx=64, dgamma=P, dbeta=P, ws=P, bytes=need, stream=None)
    _expect(lib.grem_layer_norm_backward, "type n d dy lddy x mean rstd gamma dx lddx dgamma dbeta ws bytes stream", args, [
        dict(mean=P + 2), dict(rstd=P + 2), dict(ws=P + 64), dict(dbeta=None, ws=P + 64)])


def test_a_workspace_that_is_not_used_is_not_looked_at(lib):
    order = "rowptr bits colidx nnz n labels type d x ldx out ldo counts ws bytes stream"
    args = dict(rowptr=P, bits=64, colidx=P, nnz=100, n=0, labels=P, type=F32, d=64, x=P, ldx=64, out=P, ldo=64, counts=P, ws=P + 4, bytes=4, stream=None)
    assert lib.grem_neighbour_mean_bytes(F32, 0, 100, 64, 1) == 0 and _call(lib.grem_neighbour_mean, order, args) == B.OK
