"""Host-only checks of the microscaled 4-bit operands: exports, struct layouts, sizes, refusals (no kernel is launched), and the
64-bit model that the GPU tests compare with against hand-worked blocks."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import mx_refmodel as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BASE = 0x7F0000000000           # well-aligned addresses that are never followed


@pytest.fixture(scope="module")
def X():
    from paper_2512_22804_amd import binding, build, mx
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return mx


def test_exports_every_declared_symbol(X):
    text = open(os.path.join(ROOT, "include", "mor_mx.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(mor_(?:mx|expert)_[a-z_0-9]+)\s*\(", text))
    assert names == set(X.EXPORTS)
    for n in names:
        assert getattr(X.load(), n) is not None


def test_struct_layouts(X):
    assert C.sizeof(X.MorMxOperand) == 48 and C.sizeof(X.MorMxParams) == 56 and C.sizeof(X.MorExpertOrder) == 48


def test_capacity(X):
    assert X.expert_capacity(0, 2, 8) == 0
    assert X.expert_capacity(1, 1, 8) == 128
    assert X.expert_capacity(1, 1, 8, align=1) == 1
    assert X.expert_capacity(10, 2, 4, align=128) == 640            # 20 + 4 * 127, to whole segments
    assert X.expert_capacity(8192, 2, 16, align=128) == 18432 and X.expert_capacity(3, 1, 8, align=32) == 96
    for tokens, top_k, experts, align in ((-1, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1025, 1), (1, 1, 1, 0), (1 << 24, 2, 4, 1)):
        assert X.expert_capacity(tokens, top_k, experts, align=align) == -1


def operand(X, rows, cols, **over):
    blocks = -(-cols // 32)
    o = X.MorMxOperand(BASE, 16 * blocks, BASE + (1 << 34), -(-blocks // 4) * 4, 0, 0)
    for k, v in over.items():
        setattr(o, k, v)
    return C.byref(o)


def order(X, tokens=4, top_k=2, experts=3, align=128, **over):
    o = X.MorExpertOrder(tokens, top_k, experts, align, max(0, X.expert_capacity(tokens, top_k, experts, align)), 0, BASE, BASE + 4096,
                         BASE + 8192)
    for k, v in over.items():
        setattr(o, k, v)
    return C.byref(o)


def test_quantize_refusals(X):
    lib = X.load()

    def call(rows=64, cols=96, x=BASE, out="yes", out_t=None, order=None, weights=None, **over):
        p = X.MorMxParams(rows, cols, cols, 1, 0, 0, 0, 0)
        for k, v in over.items():
            setattr(p, k, v)
        out = operand(X, rows, cols) if out == "yes" else out
        return lib.mor_mx_quantize(C.byref(p), x, out, out_t, order, weights, None)

    assert lib.mor_mx_quantize(None, BASE, operand(X, 1, 1), None, None, None, None) == 1
    assert call(out=None) == 1                                              # neither form
    assert call(x=None) == 1
    assert call(out=operand(X, 64, 96, codes=None)) == 1
    assert call(out=operand(X, 64, 96, scales=None)) == 1
    assert call(x=BASE + 1) == 3
    assert call(ld=95) == 2
    assert call(rows=-1) == 2 and call(cols=0) == 2 and call(batch=0) == 2 and call(batch=65536) == 2
    assert call(scale_rule=2) == 4 and call(rounding=2) == 4
    assert call(out=operand(X, 64, 96, ld_codes=32)) == 2                   # shorter than three blocks
    assert call(out=operand(X, 64, 96, ld_codes=56)) == 3
    assert call(out=operand(X, 64, 96, codes=BASE + 8)) == 3
    assert call(out=operand(X, 64, 96, ld_scales=2)) == 2
    assert call(out=operand(X, 64, 96, ld_scales=6)) == 3
    assert call(out=operand(X, 64, 96, scales=BASE + 2)) == 3
    assert call(out_t=operand(X, 96, 32)) == 2                              # the transpose needs two blocks
    assert call(batch=2, out=operand(X, 64, 96, batch_codes=8)) == 3
    assert call(weights=BASE) == 4                                          # weights without an order
    assert call(rows=4, order=order(X), batch=2) == 4
    assert call(rows=5, order=order(X)) == 2                                # not the order's tokens
    assert call(rows=4, order=order(X, capacity=128)) == 2                  # fewer slots than the order may take
    assert call(rows=4, order=order(X), weights=BASE + 2) == 3
    assert call(rows=0) == 0                                                # nothing to do


def test_product_refusals(X):
    lib = X.load()

    def call(m=8, n=8, k=64, a="yes", b="yes", c=BASE, ld=8, t=0, ws=None, nbytes=0):
        a = operand(X, m, k) if a == "yes" else a
        b = operand(X, n, k) if b == "yes" else b
        return lib.mor_mx_product(m, n, k, a, b, c, ld, t, ws, nbytes, None)

    assert call(a=None) == 1 and call(b=None) == 1 and call(c=None) == 1
    assert call(m=-1) == 2 and call(k=0) == 2 and call(ld=7) == 2
    assert call(c=BASE + 1) == 3 and call(c=BASE + 2, t=1) == 3
    assert call(t=2) == 4
    assert call(b=operand(X, 8, 32)) == 2
    assert call(m=0) == 0 and call(n=0) == 0
    for m, n, k in ((0, 8, 64), (8, 0, 64), (-1, 8, 64), (8, 8, 0)):
        assert X.mor_mx_product_workspace_bytes(m, n, k) == 0
    rows = lambda o, a=None, b=None, c=BASE, n=8, k=64, ld=8, t=0: lib.mor_mx_product_rows(
        n, k, a or operand(X, 512, k), b or operand(X, n, k, batch_codes=256, batch_scales=32), o, c, ld, t, None)
    assert rows(None) == 1 and rows(order(X), c=None) == 1
    assert rows(order(X, align=0)) == 2 and rows(order(X, reserved=1)) == 2 and rows(order(X, capacity=511)) == 2
    assert rows(order(X, offsets=None)) == 1 and rows(order(X, offsets=BASE + 2)) == 3
    assert rows(order(X), ld=4) == 2 and rows(order(X), t=7) == 4 and rows(order(X), k=0) == 2
    assert rows(order(X), b=operand(X, 8, 64, batch_codes=24)) == 3
    assert rows(order(X, tokens=0, capacity=0)) == 0
    depth = lambda o, cap, t=0, c=BASE, ld=8: lib.mor_mx_product_depth(8, 8, operand(X, 8, cap), operand(X, 8, cap), o, c, ld, 64, t, None)
    assert depth(order(X, align=32), 512) == 4                              # segments are no whole steps
    assert depth(order(X), 64) == 2                                         # operands shorter than the slots
    assert depth(order(X), 1024, c=None) == 1 and depth(order(X), 1024, t=3) == 4 and depth(order(X), 1024, ld=4) == 2


def test_expert_refusals(X):
    lib = X.load()
    assert lib.mor_expert_sort(None, order(X), None, 0, None) == 1
    assert lib.mor_expert_sort(BASE, None, None, 0, None) == 1
    assert lib.mor_expert_sort(BASE + 2, order(X), None, 0, None) == 3
    big = order(X, tokens=8192)
    assert X.load().mor_expert_workspace_bytes(8192, 2, 3) > 0
    assert lib.mor_expert_sort(BASE, big, None, 0, None) == 5
    assert lib.mor_expert_sort(BASE, big, BASE + 4, 1 << 20, None) == 3
    assert lib.mor_expert_sort(BASE, order(X, slot_of=None), None, 0, None) == 1
    assert lib.mor_expert_gather(BASE, 8, 0, order(X), BASE, 8, None) == 2
    assert lib.mor_expert_gather(BASE, 7, 8, order(X), BASE, 8, None) == 2
    assert lib.mor_expert_gather(BASE, 8, 8, order(X), None, 8, None) == 1
    assert lib.mor_expert_gather(BASE + 1, 8, 8, order(X), BASE, 8, None) == 3
    assert lib.mor_expert_combine(None, 8, 8, order(X), None, BASE, 8, None) == 1
    assert lib.mor_expert_combine(BASE, 8, 8, order(X), BASE + 2, BASE, 8, None) == 3
    assert lib.mor_expert_combine(BASE, 4, 8, order(X), None, BASE, 8, None) == 2
    back = lambda **k: lib.mor_expert_combine_backward(*{**dict(dy=BASE, ld_dy=8, ys=BASE, ld_ys=8, d=8, o=order(X), w=BASE, dys=BASE, ld_dys=8,
                                                                dw=BASE, st=None), **k}.values())
    assert back(dy=None) == 1 and back(ys=None) == 1 and back(w=None) == 1 and back(dys=None, dw=None) == 1
    assert back(ld_dys=7) == 2 and back(d=0) == 2 and back(dw=BASE + 2) == 3


def test_binding_refuses_what_the_library_cannot_see(X):
    codes, scales = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)
    op = X.MxOperand(codes, scales, 4, 64)
    assert op.blocks == 2 and op.batch == 1
    with pytest.raises(ValueError):
        X.MxOperand(codes, scales, 4, 65)                                   # codes too short
    with pytest.raises(ValueError):
        X.MxOperand(codes.to(torch.int8), scales, 4, 64)
    with pytest.raises(ValueError):
        X.MxOperand(codes, scales[:3], 4, 64)
    with pytest.raises(ValueError):
        X.mor_mx_quantize(torch.zeros(4, 64, dtype=torch.bfloat16), op)     # host memory
    with pytest.raises(ValueError):
        X.mor_mx_product(op, op, torch.zeros(4, 4))


# ---- the model, by hand ------------------------------------------------------------------------------------------------

def test_model_rounding_and_ties():
    x = np.zeros((1, 32))
    x[0, :15] = [4.0, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 6.0, 7.5, -0.0, -0.3, 0.2]
    codes, scales, values = R.quantize(x)
    assert scales[0, 0] == 127                                              # amax 7.5: floor(log2) - 2 = 0
    assert values[0, :15].tolist() == [4.0, 0.0, 0.5, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0, 6.0, 0.0, -0.5, 0.0]
    assert codes[0, :15].tolist() == [6, 0, 1, 2, 2, 4, 4, 6, 6, 7, 7, 7, 8, 9, 0]
    codes, scales, values = R.quantize(x, "ceil")
    assert scales[0, 0] == 128 and values[0, 11] == 8.0                     # 7.5 / 2 = 3.75 -> 4
    x[0, 11] = 6.0
    assert R.quantize(x, "ceil")[1][0, 0] == 127                            # 6 itself fits


def test_model_scales_at_the_ends():
    x = np.zeros((5, 32))
    x[1, 3] = 2.0 ** -133                                                   # smallest BF16
    x[2, 3] = 255 / 128 * 2.0 ** 127                                        # largest
    x[3, 3] = np.inf
    x[4, 3] = np.nan
    _, scales, values = R.quantize(x)
    assert scales[:, 0].tolist() == [127, 0, 252, 255, 255]
    assert values[2, 3] == 6.0 * 2.0 ** 125 and np.isnan(values[3:]).all() and values[1, 3] == 0.0
    assert R.quantize(x, "ceil")[1][:, 0].tolist() == [127, 0, 253, 255, 255]


def test_model_stochastic_is_unbiased_and_keeps_grid_values():
    n = 1 << 16
    x = np.tile(np.array([[4.0, 0.1, 1.3, 2.25, 5.0, -3.75, 1.5, 3.0]]), (n, 4))
    r = R.random16(n, 32, 0, 12345)
    _, _, values = R.quantize(x, "floor", r)
    assert set(np.unique(values[:, 0])) == {4.0} and set(np.unique(values[:, 6])) == {1.5} and set(np.unique(values[:, 7])) == {3.0}
    # mean of n draws of variance below step^2 / 4: six standard errors
    for j, step in ((1, 0.5), (2, 0.5), (3, 1.0), (4, 2.0), (5, 1.0)):
        assert abs(values[:, j].mean() - x[0, j]) < 6 * step / 2 / np.sqrt(n)
    assert not np.array_equal(R.random16(4, 32, 0, 1), R.random16(4, 32, 1, 1))
    assert not np.array_equal(R.random16(4, 32, 0, 1), R.random16(4, 32, 0, 1 << 32 | 1))
    assert not np.array_equal(R.random16(4, 32, 0, 1, batch=0), R.random16(4, 32, 0, 1, batch=1))


def test_model_sort():
    ids = np.array([[2, 0], [2, -1], [0, 2]], np.int32)
    starts, slot, src = R.sort(ids, 4, 4, 16)
    assert starts.tolist() == [0, 4, 4, 8, 8]
    assert slot.tolist() == [4, 0, 5, -1, 1, 6]
    assert src.tolist() == [1, 4, -1, -1, 0, 2, 5, -1] + [-1] * 8
