"""Tokens sorted by expert, rows gathered and added up, their gradients, and the products over the experts, against the
64-bit model.

Sums over top_k terms run in binary32 in a fixed order: within (top_k + 1) 2^-24 of sum |terms|, then half a BF16 unit (2^-9 of
the result, 2^-8 allowed near a power of two).  Scalar products of d terms: within d 2^-24 of sum |terms| whatever the order.
Weighted operands are quantised from the binary32 product, which the model forms too, so codes are equal.
"""
import numpy as np
import pytest
import torch

import mx_refmodel as R
from paper_2512_22804_amd import mx
from test_gpu_mx import bf16, check_operand, close, guarded, operand_values, random_operand

pytestmark = pytest.mark.gpu
DEV = "cuda"


def routing(tokens, top_k, experts, seed, drop=0.1, skew=0.0):
    rng = np.random.default_rng(seed)
    p = np.exp(skew * rng.standard_normal(experts))
    ids = rng.choice(experts, size=(tokens, top_k), p=p / p.sum()).astype(np.int32)
    ids[rng.random(ids.shape) < drop] = -1
    return ids


def make_order(ids, experts, align):
    order = mx.alloc_order(*ids.shape, experts, DEV, align=align)
    for t in (order.offsets, order.slot_of, order.src):
        t.fill_(-7)
    if order.workspace is not None:
        order.workspace.fill_(0xFF)
    mx.mor_expert_sort(torch.from_numpy(ids).to(DEV), order)
    return order


ORDERS = [(1, 1, 1, 1, 0.0), (1, 1, 8, 128, 0.0), (7, 2, 3, 1, 0.2), (64, 4, 60, 32, 0.0), (333, 4, 32, 1, 0.05), (1000, 1, 1024, 128, 0.1),
          (513, 8, 256, 16, 0.0), (2048, 2, 4, 128, 0.0), (2049, 2, 7, 128, 0.5), (5000, 3, 129, 1, 0.1), (20000, 2, 16, 128, 0.01),
          (9, 2, 5, 128, 1.0)]


@pytest.mark.parametrize("tokens, top_k, experts, align, drop", ORDERS)
def test_sort(tokens, top_k, experts, align, drop):
    ids = routing(tokens, top_k, experts, tokens + experts, drop, skew=1.0)
    order = make_order(ids, experts, align)
    starts, slot, src = R.sort(ids, experts, align, order.capacity)
    assert np.array_equal(order.offsets.cpu().numpy(), starts)
    assert np.array_equal(order.slot_of.cpu().numpy(), slot)
    assert np.array_equal(order.src.cpu().numpy(), src)


def test_sort_everything_to_one_expert_and_strange_numbers():
    ids = np.full((3000, 2), 5, np.int32)
    ids[:, 1] = np.where(np.arange(3000) % 3 == 0, 6, np.where(np.arange(3000) % 3 == 1, -2 ** 31, 2 ** 31 - 1))
    order = make_order(ids, 6, 128)                           # 6, the least and the largest number: no experts
    starts, slot, src = R.sort(np.where(ids == 5, 5, -1), 6, 128, order.capacity)
    assert np.array_equal(order.offsets.cpu().numpy(), starts)
    assert np.array_equal(order.slot_of.cpu().numpy(), slot) and np.array_equal(order.src.cpu().numpy(), src)


def test_no_tokens():
    order = mx.alloc_order(0, 2, 4, DEV, align=128)
    order.offsets.fill_(9)
    mx.mor_expert_sort(torch.empty(0, 2, dtype=torch.int32, device=DEV), order)
    assert (order.offsets == 0).all()
    x = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    mx.mor_expert_gather(x, order, torch.empty(0, 64, dtype=torch.bfloat16, device=DEV))
    mx.mor_expert_combine(x, order, None, torch.empty(0, 64, dtype=torch.bfloat16, device=DEV))
    w = random_operand(40, 64, 1, batch=4)[0]
    xq = mx.alloc_operand(0, 64, DEV)
    mx.mor_mx_quantize(x, xq, order=order)
    mx.mor_mx_product_rows(xq, w, order, torch.empty(0, 40, device=DEV))
    a, b = mx.alloc_operand(40, 0, DEV), mx.alloc_operand(64, 0, DEV)
    dw = torch.full((4, 40, 64), 5.0, device=DEV)
    mx.mor_mx_product_depth(a, b, order, dw)
    assert (dw == 0).all()


@pytest.mark.parametrize("d, pad", [(8, 0), (1, 0), (100, 3), (1000, 8), (1031, 0), (4096, 0)])
@pytest.mark.parametrize("tokens, top_k, experts, align", [(1, 1, 4, 1), (50, 3, 7, 1), (70, 2, 5, 128)])
def test_gather_combine_and_gradients(tokens, top_k, experts, align, d, pad):
    rng = np.random.default_rng(tokens + d)
    ids = routing(tokens, top_k, experts, d, 0.15)
    if tokens > 10:
        ids[3] = -1                                            # a token without any expert
    order = make_order(ids, experts, align)
    cap = order.capacity
    starts, slot, src = R.sort(ids, experts, align, cap)
    rows = lambda n: torch.full((n, d + pad), 7.0, dtype=torch.bfloat16, device=DEV)
    x, xv = bf16(operand_values(tokens, d + pad, 1))
    ys, yv = bf16(operand_values(cap, d + pad, 2))
    dy, gv = bf16(operand_values(tokens, d + pad, 3))
    xv, yv, gv = xv[:, :d], yv[:, :d], gv[:, :d]
    weights = rng.standard_normal((tokens, top_k)).astype(np.float32)
    w = torch.from_numpy(weights).to(DEV)

    xs = rows(cap)
    mx.mor_expert_gather(x[:, :d], order, xs[:, :d])
    want = np.where((src >= 0)[:, None], xv[np.maximum(src, 0) // top_k], 0.0)
    assert np.array_equal(xs[:, :d].double().cpu().numpy(), want) and (xs[:, d:] == 7.0).all()

    slots = slot.reshape(tokens, top_k)
    picked = np.where((slots >= 0)[..., None], yv[np.maximum(slots, 0)], 0.0)
    for use in (True, False):
        y = rows(tokens)
        mx.mor_expert_combine(ys[:, :d], order, w if use else None, y[:, :d])
        terms = picked * (weights.astype(np.float64)[..., None] if use else 1.0)
        exact, total = terms.sum(1), np.abs(terms).sum(1)
        assert (np.abs(y[:, :d].double().cpu().numpy() - exact) <= (top_k + 1) * 2.0 ** -24 * total + 2.0 ** -8 * np.abs(exact)).all()
        assert (y[:, d:] == 7.0).all()

    dots = (picked * gv[:, None, :]).sum(-1)
    bound = d * 2.0 ** -24 * (np.abs(picked) * np.abs(gv[:, None, :])).sum(-1) + 2.0 ** -23 * np.abs(dots)
    scaled = np.where((src >= 0)[:, None], gv[np.maximum(src, 0) // top_k] * weights.reshape(-1).astype(np.float64)[np.maximum(src, 0)][:, None], 0.0)
    for form in ("both", "dys", "dweights"):
        dys, dw = rows(cap), torch.full((tokens, top_k), 9.0, device=DEV)
        mx.mor_expert_combine_backward(dy[:, :d], ys[:, :d], order, w, dys[:, :d] if form != "dweights" else None, dw if form != "dys" else None)
        if form != "dweights":
            assert (np.abs(dys[:, :d].double().cpu().numpy() - scaled) <= 2.0 ** -8 * np.abs(scaled)).all() and (dys[:, d:] == 7.0).all()
        if form != "dys":
            assert (np.abs(dw.double().cpu().numpy() - dots) <= bound).all()
            assert (dw.cpu().numpy()[slots < 0] == 0).all()


def test_gradients_against_differences():
    """f = <dy, combine(ys, weights)> on small whole numbers, where every sum is exact in BF16: the gradient of f in each
    routing weight is its difference quotient, and so is the one in each row's elements."""
    tokens, top_k, experts, d = 12, 2, 4, 16
    rng = np.random.default_rng(0)
    ids = routing(tokens, top_k, experts, 3, 0.2)
    order = make_order(ids, experts, 4)
    ys = torch.from_numpy(rng.integers(-3, 4, (order.capacity, d)).astype(np.float32)).to(DEV, torch.bfloat16)
    dy = torch.from_numpy(rng.integers(-2, 3, (tokens, d)).astype(np.float32)).to(DEV, torch.bfloat16)
    w = torch.from_numpy(rng.integers(1, 4, (tokens, top_k)).astype(np.float32)).to(DEV)

    def f(ys, w):
        y = torch.empty(tokens, d, dtype=torch.bfloat16, device=DEV)
        mx.mor_expert_combine(ys, order, w, y)
        return float((y.double() * dy.double()).sum())

    dys, dw = torch.empty_like(ys), torch.empty_like(w)
    mx.mor_expert_combine_backward(dy, ys, order, w, dys, dw)
    for t in range(tokens):
        for j in range(top_k):
            up, down = w.clone(), w.clone()
            up[t, j] += 1
            down[t, j] -= 1
            assert float(dw[t, j]) == (f(ys, up) - f(ys, down)) / 2
    for s in range(0, order.capacity, 3):
        for c in (0, 7, 15):
            up, down = ys.clone(), ys.clone()
            up[s, c] += 1
            down[s, c] -= 1
            assert float(dys[s, c]) == (f(up, w) - f(down, w)) / 2


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("tokens, top_k, experts, align, d", [(1, 1, 4, 1, 40), (90, 2, 5, 1, 200), (70, 3, 6, 128, 133)])
def test_quantize_sorted_rows(tokens, top_k, experts, align, d, weighted, rounding):
    ids = routing(tokens, top_k, experts, d, 0.1)
    order = make_order(ids, experts, align)
    cap = order.capacity
    _, _, src = R.sort(ids, experts, align, cap)
    x, v = bf16(operand_values(tokens, d, 4))
    weights = np.random.default_rng(1).standard_normal((tokens, top_k)).astype(np.float32)
    rows = v[np.maximum(src, 0) // top_k]
    if weighted:
        rows = (rows.astype(np.float32) * weights.reshape(-1)[np.maximum(src, 0)][:, None]).astype(np.float64)
    rows = np.where((src >= 0)[:, None], rows, 0.0)
    random = (lambda r, c, form: R.random16(r, c, form, 17)) if rounding == "stochastic" else (lambda *a: None)
    for form in ("both", "rows", "cols"):
        out = guarded(cap, d) if form != "cols" else None
        out_t = guarded(d, cap) if form != "rows" else None
        mx.mor_mx_quantize(x, out, out_t, order=order, weights=torch.from_numpy(weights).to(DEV) if weighted else None, rounding=rounding, seed=17)
        if out is not None:
            check_operand(out, *R.quantize(rows, "floor", random(cap, d, 0))[:2])
        if out_t is not None:
            check_operand(out_t, *R.quantize(rows.T, "floor", random(d, cap, 1))[:2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens, top_k, experts, align, n, k", [(1, 1, 1, 1, 40, 64), (1, 2, 64, 1, 256, 512), (4, 4, 64, 1, 300, 100),
                                                                   (100, 2, 5, 1, 33, 257), (300, 2, 3, 128, 130, 640), (700, 1, 8, 128, 512, 300),
                                                                   (600, 4, 100, 1, 70, 128)])
def test_product_rows(tokens, top_k, experts, align, n, k, dtype):
    print(f"[mx] product_rows {tokens}x{top_k} over {experts}, align {align}, {n}x{k} {dtype}", flush=True)
    ids = routing(tokens, top_k, experts, n, 0.05, skew=1.5)
    order = make_order(ids, experts, align)
    starts, _, _ = R.sort(ids, experts, align, order.capacity)
    a, av = random_operand(order.capacity, k, 1)
    b, bv = random_operand(n, k, 2, batch=experts)
    c = torch.full((order.capacity + 1, n + 3), 7.0, dtype=dtype, device=DEV)
    mx.mor_mx_product_rows(a, b, order, c[:-1, :n])
    got = c.double().cpu().numpy()
    assert (got[:, n:] == 7.0).all() and (got[starts[-1]:] == 7.0).all()
    for e in range(experts):
        s = slice(starts[e], starts[e + 1])
        if starts[e] < starts[e + 1]:
            close(got[s, :n], av[s], bv[e], dtype == torch.float32, k)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens, top_k, experts, align, m, n", [(1, 1, 1, 128, 40, 64), (1, 2, 9, 128, 33, 130), (300, 2, 3, 128, 130, 257),
                                                                   (900, 1, 8, 256, 512, 260), (1500, 2, 4, 128, 100, 70)])
def test_product_depth(tokens, top_k, experts, align, m, n, dtype):
    print(f"[mx] product_depth {tokens}x{top_k} over {experts}, align {align}, {m}x{n} {dtype}", flush=True)
    ids = routing(tokens, top_k, experts, n, 0.05, skew=1.5)
    ids[ids == experts - 1] = 0                                # an expert without a token, unless it is the only one
    order = make_order(ids, experts, align)
    cap = order.capacity
    starts, _, _ = R.sort(ids, experts, align, cap)
    a, av = random_operand(m, cap, 1)
    b, bv = random_operand(n, cap, 2)
    a.scales[:, starts[-1] // 32:] = 255                       # behind the last segment: read by nobody
    c = torch.full((experts, m + 1, n + 5), 7.0, dtype=dtype, device=DEV)
    mx.mor_mx_product_depth(a, b, order, c[:, :m, :n])
    got = c.double().cpu().numpy()
    assert (got[:, m:] == 7.0).all() and (got[:, :, n:] == 7.0).all()
    for e in range(experts):
        s = slice(starts[e], starts[e + 1])
        close(got[e, :m, :n], av[:, s], bv[:, s], dtype == torch.float32, max(1, starts[e + 1] - starts[e]))


def test_an_expert_layer_forward_and_backward():
    """Sort, gather and quantise, product, weighted sum, and back, on whole numbers that four bits hold exactly: everything
    equals the layer in binary64."""
    tokens, top_k, experts, d, n = 200, 2, 6, 64, 96
    rng = np.random.default_rng(5)
    exact_grid = lambda *s: rng.choice([-2.0, -1.0, 0.0, 1.0, 2.0, 4.0], s)   # amax 4 (or 2, 1): every block exact
    ids = routing(tokens, top_k, experts, 1, 0.1)
    order = make_order(ids, experts, 128)
    x, xv = bf16(exact_grid(tokens, d))
    w, wv = bf16(exact_grid(experts, n, d))
    dy, gv = bf16(exact_grid(tokens, n))
    weights = rng.choice([0.5, 1.0], (tokens, top_k)).astype(np.float32)      # weighted: 0.5 .. 4, still exact
    r = torch.from_numpy(weights).to(DEV)
    cap = order.capacity
    xq, xqt = mx.alloc_operand(cap, d, DEV), mx.alloc_operand(d, cap, DEV)
    wq, wqt = mx.alloc_operand(n, d, DEV, batch=experts), mx.alloc_operand(d, n, DEV, batch=experts)
    mx.mor_mx_quantize(x, xq, xqt, order=order)
    mx.mor_mx_quantize(w, wq, wqt)
    ys = torch.empty(cap, n, dtype=torch.bfloat16, device=DEV)
    y = torch.empty(tokens, n, dtype=torch.bfloat16, device=DEV)
    mx.mor_mx_product_rows(xq, wq, order, ys)
    mx.mor_expert_combine(ys, order, r, y)
    hit = ids >= 0
    per = np.einsum("td,tjnd->tjn", xv, wv[np.maximum(ids, 0)]) * hit[..., None]
    per = torch.from_numpy(per).to(torch.bfloat16).double().numpy()          # the experts' results are kept in BF16
    want = torch.from_numpy((per * weights[..., None]).sum(1)).to(torch.bfloat16).double().numpy()
    assert np.array_equal(y.double().cpu().numpy(), want)
    gq, gqt = mx.alloc_operand(cap, n, DEV), mx.alloc_operand(n, cap, DEV)
    mx.mor_mx_quantize(dy, gq, gqt, order=order, weights=r)
    dxs = torch.empty(cap, d, device=DEV)
    dw = torch.empty(experts, n, d, device=DEV)
    mx.mor_mx_product_rows(gq, wqt, order, dxs)
    mx.mor_mx_product_depth(gqt, xqt, order, dw)
    slots = order.slot_of.cpu().numpy().reshape(tokens, top_k)
    back = np.einsum("tn,tjnd->tjd", gv, wv[np.maximum(ids, 0)]) * weights[..., None]
    got = dxs.double().cpu().numpy()[np.maximum(slots, 0)]
    assert np.array_equal(got[hit], back[hit])
    want = np.zeros((experts, n, d))
    for t in range(tokens):
        for j in range(top_k):
            if hit[t, j]:
                want[ids[t, j]] += weights[t, j] * np.outer(gv[t], xv[t])
    assert np.array_equal(dw.double().cpu().numpy(), want)
