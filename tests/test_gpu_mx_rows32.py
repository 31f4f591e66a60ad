"""Experts' rows in binary32, added up and their gradients, against the 64-bit model.

Sums over top_k terms run in binary32 in a fixed order: within (top_k + 1) 2^-24 of sum |terms|, then half a unit of the result's type
(2^-24 of it, or for BF16 2^-8 as for rows in BF16).  Scalar products of d terms: within d 2^-24 of sum |terms| whatever the order."""
import numpy as np
import pytest
import torch

import mx_refmodel as R
from paper_2512_22804_amd import binding as B
from paper_2512_22804_amd import mx
from test_gpu_mx import bf16, operand_values
from test_gpu_mx_experts import make_order, routing

pytestmark = pytest.mark.gpu
DEV = "cuda"


def f32(values):
    t = torch.from_numpy(np.ascontiguousarray(values, dtype=np.float32))
    return t.to(DEV), t.double().numpy()


@pytest.mark.parametrize("d, pad", [(8, 0), (1, 0), (100, 3), (1000, 8), (1031, 0), (4096, 0)])
@pytest.mark.parametrize("tokens, top_k, experts, align", [(1, 1, 4, 1), (50, 3, 7, 1), (70, 2, 5, 128), (33, 9, 12, 1)])
def test_combine_and_gradients(tokens, top_k, experts, align, d, pad):
    rng = np.random.default_rng(tokens + d)
    ids = routing(tokens, top_k, experts, d, 0.15)
    if tokens > 10:
        ids[3] = -1                                            # a token without any expert
    order = make_order(ids, experts, align)
    cap = order.capacity
    _, slot, src = R.sort(ids, experts, align, cap)
    ys, yv = f32(operand_values(cap, d + pad, 2))
    dy, gv = bf16(operand_values(tokens, d + pad, 3))
    yv, gv = yv[:, :d], gv[:, :d]
    weights = rng.standard_normal((tokens, top_k)).astype(np.float32)
    w = torch.from_numpy(weights).to(DEV)
    slots = slot.reshape(tokens, top_k)
    picked = np.where((slots >= 0)[..., None], yv[np.maximum(slots, 0)], 0.0)
    for dtype, unit in ((torch.float32, 2.0 ** -24), (torch.bfloat16, 2.0 ** -8)):
        for use in (True, False):
            y = torch.full((tokens, d + pad), 7.0, dtype=dtype, device=DEV)
            mx.mor_expert_combine(ys[:, :d], order, w if use else None, y[:, :d])
            terms = picked * (weights.astype(np.float64)[..., None] if use else 1.0)
            exact, total = terms.sum(1), np.abs(terms).sum(1)
            assert (np.abs(y[:, :d].double().cpu().numpy() - exact) <= (top_k + 1) * 2.0 ** -24 * total + unit * np.abs(exact)).all()
            assert (y[:, d:] == 7.0).all()

    dots = (picked * gv[:, None, :]).sum(-1)
    bound = d * 2.0 ** -24 * (np.abs(picked) * np.abs(gv[:, None, :])).sum(-1) + 2.0 ** -23 * np.abs(dots)
    scaled = np.where((src >= 0)[:, None], gv[np.maximum(src, 0) // top_k] * weights.reshape(-1).astype(np.float64)[np.maximum(src, 0)][:, None], 0.0)
    for form in ("both", "dys", "dweights"):
        dys, dw = torch.full((cap, d + pad), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((tokens, top_k), 9.0, device=DEV)
        mx.mor_expert_combine_backward(dy[:, :d], ys[:, :d], order, w, dys[:, :d] if form != "dweights" else None, dw if form != "dys" else None)
        if form != "dweights":
            assert (np.abs(dys[:, :d].double().cpu().numpy() - scaled) <= 2.0 ** -8 * np.abs(scaled)).all() and (dys[:, d:] == 7.0).all()
        if form != "dys":
            assert (np.abs(dw.double().cpu().numpy() - dots) <= bound).all()
            assert (dw.cpu().numpy()[slots < 0] == 0).all()


def test_refusals():
    order = make_order(np.zeros((4, 2), np.int32), 3, 1)
    ys, y, w = torch.zeros(order.capacity, 16, device=DEV), torch.zeros(4, 16, device=DEV), torch.zeros(4, 2, device=DEV)
    with pytest.raises(ValueError):
        mx.mor_expert_combine(ys.bfloat16(), order, w, y)                   # rows in BF16, the sum in binary32
    with pytest.raises(ValueError):
        mx.mor_expert_combine(ys.double(), order, w, y)
    with pytest.raises(ValueError):
        mx.mor_expert_combine(ys, order, w, y[:3])
    with pytest.raises(ValueError):
        mx.mor_expert_combine_backward(y, ys, order, w, None, w)            # dy in binary32
    with pytest.raises(B.MorError):
        mx.mor_expert_combine(ys[:1].expand(order.capacity, 16), order, w, y)       # rows upon each other
    with pytest.raises(B.MorError):
        mx.mor_expert_combine_backward(y.bfloat16(), ys, order, w, None, None)
    # what only the library sees
    call = lambda ys=ys.data_ptr(), y=y.data_ptr(), t=1: mx.load().mor_expert_combine_f32(ys, 16, 16, order.struct(), None, y, 16, t, None)
    assert call(ys=ys.data_ptr() + 2) == 3 and call(y=y.data_ptr() + 2) == 3 and call(t=2) == 4 and call(ys=None) == 1 and call(y=None) == 1


def test_no_tokens():
    order = mx.alloc_order(0, 2, 4, DEV, align=128)
    mx.mor_expert_sort(torch.empty(0, 2, dtype=torch.int32, device=DEV), order)
    none = torch.empty(0, 64, device=DEV)
    mx.mor_expert_combine(none, order, None, none)
    mx.mor_expert_combine_backward(none.bfloat16(), none, order, None, None, torch.empty(0, 2, device=DEV))
