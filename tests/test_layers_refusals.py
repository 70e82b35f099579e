"""What the layer operators refuse, at the C entry points (argument checks come before any launch, so this runs without a GPU; the
pointers are never followed) and in the binding."""
import ctypes
import os

import pytest
import torch

from paper_2502_17846_amd import binding as B

P = 1 << 20                        # an aligned address that nothing reads
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2502_17846_amd import build
        build.build_library()
    return B.load()


def _call(fn, order, args, **change):
    """fn with the arguments of `args` in that order, some of them changed."""
    unknown = set(change) - set(args)
    assert not unknown, unknown
    return fn(*[{**args, **change}[k] for k in order.split()])


def _rows(data=P, stride=64, exponents=None, exponent_stride=0):
    return ctypes.byref(B.Rows(data, stride, exponents, exponent_stride))


def _expect(fn, order, args, cases, code=B.ERR_ARG):
    for change in cases:
        assert _call(fn, order, args, **change) == code, change


SIZES = [dict(type=-1), dict(type=3), dict(n=-1), dict(n=(1 << 30) + 1)]


def test_neighbour_mean(lib):
    order = "rowptr bits colidx nnz n labels type d x ldx out ldo counts ws bytes stream"
    args = dict(rowptr=P, bits=64, colidx=P, nnz=100, n=10, labels=P, type=F32, d=64, x=P, ldx=64, out=P, ldo=64, counts=P, ws=None, bytes=0,
                stream=None)
    bad = SIZES + [dict(rowptr=None), dict(bits=16), dict(colidx=None), dict(nnz=-1), dict(d=0), dict(d=(1 << 20) + 1), dict(x=None), dict(x=P + 2),
                   dict(type=BF16, x=P + 1), dict(ldx=63), dict(out=None), dict(out=P + 1), dict(ldo=0)]
    _expect(lib.grem_neighbour_mean, order, args, bad)
    need = lib.grem_neighbour_mean_bytes(F32, 10, 100_000, 64, 1)
    assert need > 0 and lib.grem_neighbour_mean_bytes(F32, 10, 100, 64, 1) == 0
    _expect(lib.grem_neighbour_mean, order, args, [dict(nnz=100_000), dict(nnz=100_000, ws=P, bytes=need - 1)], B.ERR_NOMEM)
    assert _call(lib.grem_neighbour_mean, order, args, n=0, rowptr=None, nnz=0, colidx=None, x=None, out=None) == B.OK
    order = "rowptr bits colidx nnz n labels counts type d x ldx out ldo ws bytes stream"
    _expect(lib.grem_neighbour_mean_backward, order, args, bad + [dict(counts=None)])
    assert lib.grem_neighbour_mean_bytes(F32, 10, -1, 64, 0) == 0 and lib.grem_neighbour_mean_bytes(F32, 10, 100_000, 0, 0) == 0
    # a labelling over more rows than the caches hold: their order is kept in the workspace
    assert lib.grem_neighbour_mean_bytes(BF16, 1 << 20, 100, 64, 1) > 4 << 20 and lib.grem_neighbour_mean_bytes(BF16, 1 << 20, 100, 64, 0) == 0


def test_linear(lib):
    order = "type n m a lda ka b ldb kb w ldw bias act residual ldr out ldo pre ldp stream"
    args = dict(type=BF16, n=10, m=32, a=P, lda=64, ka=64, b=P, ldb=16, kb=16, w=P, ldw=80, bias=P, act=1, residual=P, ldr=32, out=P, ldo=32, pre=P,
                ldp=32, stream=None)
    _expect(lib.grem_linear, order, args, SIZES + [
        dict(m=0), dict(m=(1 << 20) + 1), dict(ka=0), dict(kb=-1), dict(ka=(1 << 20) + 1), dict(a=None), dict(a=P + 1), dict(lda=63), dict(b=None),
        dict(ldb=15), dict(w=None), dict(ldw=79), dict(bias=P + 1), dict(act=-1), dict(act=4), dict(residual=P + 1), dict(ldr=31), dict(out=None),
        dict(ldo=31), dict(pre=P + 1), dict(ldp=31)])
    assert _call(lib.grem_linear, order, args, n=0, a=None, b=None, out=None) == B.OK


def test_linear_backward(lib):
    order = "type n m dout ldd act pre ldp a ka b kb w ldw da ldda db lddb dw lddw dbias ws bytes stream"
    need = lib.grem_linear_backward_bytes(F16, 10, 32, 64, 16, 3)
    args = dict(type=F16, n=10, m=32, dout=P, ldd=32, act=3, pre=P, ldp=32, a=_rows(), ka=64, b=_rows(stride=16), kb=16, w=P, ldw=80, da=P, ldda=64,
                db=P, lddb=16, dw=P, lddw=80, dbias=P, ws=P, bytes=need, stream=None)
    ck = dict(a=_rows(exponents=P, exponent_stride=2), b=_rows(stride=16, exponents=P, exponent_stride=1))
    _expect(lib.grem_linear_backward, order, args, SIZES + [
        dict(m=0), dict(ka=0), dict(kb=-1), dict(dout=None), dict(ldd=31), dict(act=9), dict(pre=None), dict(ldp=31), dict(a=None),
        dict(a=_rows(data=None)), dict(a=_rows(stride=63)), dict(a=_rows(data=P + 1)), dict(b=None), dict(b=_rows(stride=15)), dict(w=None), dict(ldw=79),
        dict(da=P + 1), dict(ldda=63), dict(lddb=15), dict(lddw=79), dict(dw=P + 1), dict(dbias=P + 1), dict(kb=0),
        # one of the two a checkpoint, the other not; too few exponent bytes to a row
        dict(a=ck["a"]), dict(b=ck["b"]), dict(ck, a=_rows(exponents=P, exponent_stride=1)), dict(ck, b=_rows(stride=16, exponents=P, exponent_stride=0))])
    _expect(lib.grem_linear_backward, order, args, [dict(ws=None), dict(bytes=need - 1)], B.ERR_NOMEM)
    assert _call(lib.grem_linear_backward, order, args, da=None, db=None, dw=None, dbias=None, ws=None, bytes=0) == B.OK
    assert lib.grem_linear_backward_bytes(7, 10, 32, 64, 16, 3) == 0 and lib.grem_linear_backward_bytes(F16, 10, 0, 64, 16, 3) == 0


def test_layer_norm(lib):
    order = "type n d x ldx gamma beta eps y ldy mean rstd stream"
    args = dict(type=F32, n=10, d=64, x=P, ldx=64, gamma=P, beta=P, eps=1e-5, y=P, ldy=64, mean=P, rstd=P, stream=None)
    _expect(lib.grem_layer_norm, order, args, SIZES + [
        dict(d=0), dict(d=(1 << 20) + 1), dict(x=None), dict(x=P + 2), dict(ldx=63), dict(gamma=P + 1), dict(beta=P + 2), dict(eps=-1.0),
        dict(eps=float("nan")), dict(y=None), dict(ldy=63)])
    order = "type n d dy lddy x mean rstd gamma dx lddx dgamma dbeta ws bytes stream"
    need = lib.grem_layer_norm_backward_bytes(10, 64)
    args = dict(type=F32, n=10, d=64, dy=P, lddy=64, x=_rows(), mean=P, rstd=P, gamma=P, dx=P, lddx=64, dgamma=P, dbeta=P, ws=P, bytes=need, stream=None)
    _expect(lib.grem_layer_norm_backward, order, args, SIZES + [
        dict(d=0), dict(dy=None), dict(lddy=63), dict(x=None), dict(x=_rows(data=None)), dict(x=_rows(stride=63)),
        dict(x=_rows(exponents=P, exponent_stride=1)), dict(mean=None), dict(rstd=None), dict(gamma=P + 2), dict(dx=P + 1), dict(lddx=63),
        dict(dgamma=P + 2), dict(dbeta=P + 1)])
    _expect(lib.grem_layer_norm_backward, order, args, [dict(ws=None), dict(bytes=need - 1)], B.ERR_NOMEM)


def test_checkpoint(lib):
    order = "type n d x ldx codes ldc exponents lde stream"
    args = dict(type=F32, n=10, d=65, x=P, ldx=65, codes=P, ldc=65, exponents=P, lde=3, stream=None)
    _expect(lib.grem_checkpoint_pack, order, args, SIZES + [
        dict(d=0), dict(x=None), dict(x=P + 2), dict(ldx=64), dict(codes=None), dict(ldc=64), dict(exponents=None), dict(lde=2)])
    order = "type n d x y ldy stream"
    args = dict(type=F32, n=10, d=65, x=_rows(stride=65, exponents=P, exponent_stride=3), y=P, ldy=65, stream=None)
    _expect(lib.grem_checkpoint_unpack, order, args, SIZES + [
        dict(d=0), dict(x=None), dict(x=_rows(stride=65)), dict(x=_rows(stride=64, exponents=P, exponent_stride=3)),
        dict(x=_rows(stride=65, exponents=P, exponent_stride=2)), dict(y=None), dict(y=P + 2), dict(ldy=64)])


def test_the_binding_takes_no_host_memory():
    x, w = torch.zeros((4, 8)), torch.zeros((3, 8))
    rp, ci = torch.zeros(5, dtype=torch.int32), torch.zeros(0, dtype=torch.int32)
    v = torch.zeros(4)
    for call in (lambda: B.grem_neighbour_mean(rp, ci, 4, x), lambda: B.grem_neighbour_mean_backward(rp, ci, 4, x, rp[:4]), lambda: B.grem_linear(x, w),
                 lambda: B.grem_linear_backward(torch.zeros((4, 3)), x, w), lambda: B.grem_layer_norm(x), lambda: B.grem_checkpoint_pack(x),
                 lambda: B.grem_layer_norm_backward(x, x, v, v),
                 lambda: B.grem_checkpoint_unpack(B.Checkpoint(x.char(), x[:, :1].byte(), torch.float32))):
        with pytest.raises(TypeError, match="on the GPU"):
            call()


def test_rows_too_far_apart_for_the_mean(lib):
    order = "rowptr bits colidx nnz n labels type d x ldx out ldo counts ws bytes stream"
    args = dict(rowptr=P, bits=64, colidx=P, nnz=100, n=10, labels=P, type=F32, d=64, x=P, ldx=1 << 32, out=P, ldo=64, counts=P, ws=None, bytes=0,
                stream=None)
    assert _call(lib.grem_neighbour_mean, order, args) == B.ERR_ARG
    order = "rowptr bits colidx nnz n labels counts type d x ldx out ldo ws bytes stream"
    assert _call(lib.grem_neighbour_mean_backward, order, args) == B.ERR_ARG
