"""Calls of the 4-bit operators that were refused, or taken, wrongly."""
import ctypes as C

import pytest
import torch

from paper_2512_22804_amd import mx, mx_layers

DEV = "cuda"


@pytest.mark.gpu
def test_layers_of_experts_look_at_shapes():
    """Routing weights whose number is right and whose shape is not would be another choice's."""
    x, w = torch.randn(4, 64, device=DEV), torch.randn(3, 40, 64, device=DEV)
    ids, weights = torch.randint(0, 3, (4, 2), dtype=torch.int32, device=DEV), torch.rand(4, 2, device=DEV)
    served = mx_layers.ServedExperts(w)
    for call in (lambda *a: mx_layers.experts(a[0], w, *a[1:]), served):
        assert torch.equal(call(x, ids, weights), call(x, ids, weights.reshape(-1)))
        for wrong in ((x, ids, weights.reshape(2, 4)), (x, ids, weights.t()), (x, ids, weights[:3]), (x, ids.reshape(2, 4), weights.reshape(2, 4)),
                      (x, ids.reshape(-1), weights.reshape(-1)), (x[0], ids, weights), (x[:, :32], ids, weights)):
            with pytest.raises(ValueError):
                call(*wrong)
    with pytest.raises(ValueError):
        mx_layers.ServedExperts(w[0])


@pytest.mark.gpu
def test_layers_of_experts_take_any_strides():
    """A router's tensors as they come: a part of its columns, or its rows side by side."""
    x, w = torch.randn(6, 64, device=DEV), torch.randn(3, 40, 64, device=DEV)
    ids, weights = torch.randint(0, 3, (6, 4), dtype=torch.int32, device=DEV), torch.rand(6, 4, device=DEV)
    served = mx_layers.ServedExperts(w)
    for call in (lambda *a: mx_layers.experts(a[0], w, *a[1:]), served):
        want = call(x, ids[:, :2].contiguous(), weights[:, :2].contiguous())
        assert torch.equal(call(x, ids[:, :2], weights[:, :2]), want)
        assert torch.equal(call(x, ids[:, :2].t().contiguous().t(), weights[:, :2].t().contiguous().t()), want)
