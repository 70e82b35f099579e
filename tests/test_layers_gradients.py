"""Tensors that require gradients: the layer operators' calls are not recorded, so the binding refuses them rather than return outputs
that nothing leads back from.  Tensors without memory stand for those on the GPU."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from tests.test_layers_binding import NAMES, _calls, _t, no_library  # noqa: F401  (a fixture)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_refused_unless_recording_is_off(name, no_library, monkeypatch):  # noqa: F811
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    call, tensors = _calls()[name]
    with FakeTensorMode():
        made = {k: _t(shape, t) for k, (shape, t) in tensors.items()}
        for k, v in made.items():
            if not v.is_floating_point() or name == "unpack" and k != "out":
                continue
            v.requires_grad_()
            with pytest.raises(ValueError, match="gradient"):
                call(None, **made)
            assert not [m for m in no_library.made if not m.endswith("_bytes")], k
            with torch.no_grad():
                call(None, **made)
            call(None, **{**made, k: v.detach()})
            v.requires_grad_(False)
            del no_library.made[:]
