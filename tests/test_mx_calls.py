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


def test_an_operand_of_one_row_cut_out_of_a_larger_one():
    """Its row's distance to the next is nobody's: what counts are the bytes that its blocks take."""
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.uint8)
    for cut in (slice(0, 1), slice(2, 3)):
        op = mx.MxOperand(codes[cut, :56], scales[cut, :3], 1, 96)
        assert op._struct.ld_codes % 16 == 0 and op._struct.ld_codes >= 48
        assert op._struct.ld_scales % 4 == 0 and op._struct.ld_scales >= 3


@pytest.mark.gpu
def test_an_operand_of_one_row_cut_out_of_a_larger_one_is_written_and_read():
    x = torch.randn(1, 96, device=DEV).to(torch.bfloat16)
    want, y = mx.alloc_operand(1, 96, DEV), torch.empty(1, 96, device=DEV, dtype=torch.bfloat16)
    mx.mor_mx_quantize(x, want)
    codes, scales = torch.full((4, 64), 0xA5, dtype=torch.uint8, device=DEV), torch.full((4, 8), 0xA5, dtype=torch.uint8, device=DEV)
    op = mx.MxOperand(codes[1:2, :56], scales[1:2, :3], 1, 96)
    mx.mor_mx_quantize(x, op)
    assert torch.equal(codes[1:2, :48], want.codes) and torch.equal(scales[1:2, :3], want.scales[:, :3])
    assert (codes[[0, 2, 3]] == 0xA5).all() and (scales[[0, 2, 3]] == 0xA5).all() and (codes[1, 48:] == 0xA5).all() and (scales[1, 4:] == 0xA5).all()
    mx.mor_mx_dequantize(op, y)
    back = torch.empty_like(y)
    mx.mor_mx_dequantize(want, back)
    assert torch.equal(y, back)


@pytest.mark.gpu
@pytest.mark.parametrize("how", ["rows", "both", "stochastic"])
def test_slots_without_tokens_are_quantised(how):
    """An order of fixed capacity and no tokens: x has no address, every slot holds zeros."""
    capacity, d = 256, 64
    ints = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)
    order = mx.ExpertOrder(0, 2, 3, 128, capacity, ints(4), ints(0), ints(capacity), None)
    mx.mor_expert_sort(ints(0).view(0, 2), order)
    out = mx.alloc_operand(capacity, d, DEV)
    out_t = mx.alloc_operand(d, capacity, DEV) if how != "rows" else None
    for op in (out, out_t):
        if op is not None:
            op.codes.fill_(0xA5)
    mx.mor_mx_quantize(torch.empty(0, d, dtype=torch.bfloat16, device=DEV), out, out_t, order=order,
                       rounding="stochastic" if how == "stochastic" else "nearest")
    assert all((op.codes == 0).all() and (op.scales[:, :op.blocks] == 127).all() for op in (out, out_t) if op is not None)


def test_slots_without_tokens_need_no_tokens_address():
    """(No kernel is launched: what is refused is the operand, looked at behind x.)"""
    at = 1 << 40
    order = mx.MorExpertOrder(0, 2, 3, 128, 128, 0, at, None, at)
    params = mx.MorMxParams(0, 32, 32, 1, 0, 0, 0, 0)
    out = mx.MorMxOperand(at + 8, 16, at, 4, 0, 0)
    assert mx.load().mor_mx_quantize(C.byref(params), None, C.byref(out), None, C.byref(order), None, None) == 3
    order.tokens = params.rows = 1
    order.slot_of = at
    order.capacity = 256
    assert mx.load().mor_mx_quantize(C.byref(params), None, C.byref(out), None, C.byref(order), None, None) == 1
