"""Tensors of several devices, or of one that is not the current device, are refused by the
fine-tuning operators before anything is launched; so is what is no tensor.  (Stand-ins for CUDA
tensors: no GPU is needed.)"""
import pytest
import torch

import paper_1512_06473_gb300 as q
from paper_1512_06473_gb300 import finetune


class OnDevice(torch.Tensor):
    """A host tensor that says it is on a CUDA device."""

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return self.at


def _on(device, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice)
    t.at = device
    return t


@pytest.fixture(autouse=True)
def current_device(monkeypatch):
    monkeypatch.setattr(finetune, "_device", lambda: 0)
    monkeypatch.setattr(finetune, "load", lambda: pytest.fail("the call went on to the library"))


X, W, Y, T, B, L = (12, 16), (10, 16), (12, 10), (12,), (10,), (12,)
I64 = torch.int64
FORWARD = [("x", X, {}), ("weight", W, {}), ("bias", B, {}), ("residual", Y, {}), ("out", Y, {})]
BACKWARD = [("dy", Y, {}), ("x", X, {}), ("weight", W, {}), ("pre", Y, {})]
XENT = [("x", X, {}), ("weight", W, {}), ("targets", T, {"dtype": I64}), ("bias", B, {})]
CALLS = [("dense_forward", FORWARD, {}), ("dense_backward", BACKWARD, {"act": "relu"}), ("xent_forward", XENT, {}),
         ("xent_grad", XENT + [("dloss", L, {})], {}), ("orthogonalize", [("g", X, {}), ("out", X, {})], {})]


@pytest.mark.parametrize("name,args,more", CALLS, ids=[c[0] for c in CALLS])
def test_another_device_is_refused(name, args, more):
    for other in [a[0] for a in args]:
        given = {n: _on(int(n == other), *shape, **kw) for n, shape, kw in args}
        with pytest.raises(ValueError, match="device"):
            getattr(q, name)(**given, **more)
    # all on one device, but not the current one
    with pytest.raises(ValueError, match="device"):
        getattr(q, name)(**{n: _on(1, *shape, **kw) for n, shape, kw in args}, **more)


@pytest.mark.parametrize("name,args,more", CALLS, ids=[c[0] for c in CALLS])
def test_what_is_no_tensor_is_refused(name, args, more):
    for bad in [a[0] for a in args]:
        given = {n: [0.0] if n == bad else _on(0, *shape, **kw) for n, shape, kw in args}
        with pytest.raises(TypeError, match=bad):
            getattr(q, name)(**given, **more)
