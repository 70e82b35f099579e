"""What the binding of the layer operators refuses before it calls the library: tensors of several devices, a stream of another device, and
tensors whose gradients it would lose.  Tensors without memory stand for those on the GPU; the library is never called."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2502_17846_amd import binding as B

N, D, M = 6, 32, 5


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    """A library whose calls only say where they went."""
    class Calls:
        def __init__(self):
            self.made = []

        def __getattr__(self, name):
            def call(*args):
                self.made.append(name)
                return 0
            return call

    calls = Calls()
    monkeypatch.setattr(B, "load", lambda: calls)
    monkeypatch.setattr(B, "_raw_stream", lambda index: 0)
    return calls


def _t(shape, dtype=torch.float32, device="cuda:0"):
    return torch.empty(shape, dtype=dtype, device=device)


def _calls():
    """name: (function, its tensors)"""
    i32, f32 = torch.int32, torch.float32
    graph = dict(rp=((N + 1,), i32), ci=((20,), i32), labels=((N,), i32), x=((N, D), f32), out=((N, D), f32))
    lin = dict(a=((N, D), f32), w=((M, 2 * D), f32), bias=((M,), f32), b=((N, D), f32), residual=((N, M), f32), out=((N, M), f32))
    back = dict(dout=((N, M), f32), a=((N, D), f32), w=((M, 2 * D), f32), b=((N, D), f32), pre=((N, M), f32))
    rows = dict(mean=((N,), f32), rstd=((N,), f32), gamma=((D,), f32))
    return {
        "mean": (lambda s, rp, ci, labels, x, out: B.grem_neighbour_mean(rp, ci, N, x, labels, out, stream=s), graph),
        "mean backward": (lambda s, rp, ci, labels, x, out, counts: B.grem_neighbour_mean_backward(rp, ci, N, x, counts, labels, out, stream=s),
                          dict(graph, counts=((N,), i32))),
        "linear": (lambda s, a, w, bias, b, residual, out: B.grem_linear(a, w, bias, b, B.ACT_RELU, residual, out, stream=s), lin),
        "linear backward": (lambda s, dout, a, w, b, pre: B.grem_linear_backward(dout, a, w, b, B.ACT_RELU, pre, stream=s), back),
        "norm": (lambda s, x, gamma, beta, out: B.grem_layer_norm(x, gamma, beta, out=out, stream=s),
                 dict(x=((N, D), f32), gamma=((D,), f32), beta=((D,), f32), out=((N, D), f32))),
        "norm backward": (lambda s, dy, x, dx, **p: B.grem_layer_norm_backward(dy, x, dx=dx, stream=s, **p),
                          dict(dy=((N, D), f32), x=((N, D), f32), dx=((N, D), f32), **rows)),
        "norm backward from 8 bits": (
            lambda s, dy, codes, exponents, **p: B.grem_layer_norm_backward(dy, B.Checkpoint(codes, exponents, f32), stream=s, **p),
            dict(dy=((N, D), f32), codes=((N, D), torch.int8), exponents=((N, 1), torch.uint8), **rows)),
        "pack": (lambda s, x: B.grem_checkpoint_pack(x, stream=s), dict(x=((N, D), f32))),
        "unpack": (lambda s, codes, exponents, out: B.grem_checkpoint_unpack(B.Checkpoint(codes, exponents, f32), out, stream=s),
                   dict(codes=((N, D), torch.int8), exponents=((N, 1), torch.uint8), out=((N, D), f32))),
    }


NAMES = ["mean", "mean backward", "linear", "linear backward", "norm", "norm backward", "norm backward from 8 bits", "pack", "unpack"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_tensors_of_two_devices(name, no_library, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    call, tensors = _calls()[name]
    with FakeTensorMode():
        def made(**other):
            return {k: _t(shape, t, other.get(k, "cuda:0")) for k, (shape, t) in tensors.items()}

        call(None, **made())
        assert no_library.made
        del no_library.made[:]
        for k in tensors if len(tensors) > 1 else ():
            with pytest.raises(ValueError, match="is on cuda:"):
                call(None, **made(**{k: "cuda:1"}))
        assert not [m for m in no_library.made if not m.endswith("_bytes")]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_a_device_that_is_not_the_current_one(name, no_library, monkeypatch):
    # the launch is made with the tensors' device as the current one
    at = []

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            at.append(self.index)

        def __exit__(self, *a):
            at.append("back")

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    call, tensors = _calls()[name]
    with FakeTensorMode():
        call(None, **{k: _t(shape, t, "cuda:1") for k, (shape, t) in tensors.items()})
        assert at == [1, "back"]


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_device(name, monkeypatch):
    class Stream:
        cuda_stream, device_index, device = 0, 1, torch.device("cuda:1")

    call, tensors = _calls()[name]
    with FakeTensorMode():
        with pytest.raises(ValueError, match="stream"):
            call(Stream(), **{k: _t(shape, t) for k, (shape, t) in tensors.items()})
