"""A linear layer and a layer of experts in microscaled 4 bits, forward, backward and served, against the 64-bit model.

The model quantises the same BF16 (weighted: binary32) values, gradients with the same random bits, so all operands are equal and what
is left are the products' sums and the roundings that follow:
  a product's element       (k / 128 + 2) 2^-22 sum |terms|, then half a BF16 unit (2^-8 of it allowed) or a binary32 unit
  the layer's output        its rows are kept in BF16: those bounds and 2^-8 of every row, times the weights, then again half a unit
  weights' gradients        scalar products with rows in BF16: 2^-8 |dy| |ys| each, and the sums' 2^-24 d
"""
import ctypes as C

import numpy as np
import pytest
import torch

import mx_refmodel as R
from paper_2512_22804_amd import binding, mx, mx_layers

DEV = "cuda"


def numbers(t):
    return t.detach().double().cpu().numpy()


def made(*shape, seed, scale=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).mul_(scale).to(torch.bfloat16)


def forms(x, rule, seed=None):
    """Values of an operand and of its transpose."""
    noise = (lambda r, c, form: None) if seed is None else (lambda r, c, form: R.random16(r, c, form, seed))
    return R.quantize(x, rule, noise(*x.shape, 0))[2], R.quantize(x.T.copy(), rule, noise(*x.shape[::-1], 1))[2].T


def sums_bound(a, b):
    return (a.shape[1] / 128 + 2) * 2.0 ** -22 * (np.abs(a) @ np.abs(b).T)


def check(got, want, bound, f32=False):
    off = np.abs(numbers(got) - want) > bound + np.abs(want) * (2.0 ** -23 if f32 else 2.0 ** -8)
    assert not off.any(), f"{off.sum()} of {off.size} off, first at {np.argwhere(off)[0]}"


# ---- without a GPU -----------------------------------------------------------------------------------------------------

def test_refusals():
    x = torch.zeros(4, 32)
    with pytest.raises(ValueError):
        mx_layers.linear(x.half(), x)
    with pytest.raises(ValueError):
        mx_layers.linear(x, torch.zeros(4, 33))
    with pytest.raises(ValueError):
        mx_layers.experts(x, x, torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 1))
    with pytest.raises(ValueError):
        mx_layers.linear(x, x)                                              # host memory


def test_operands_and_orders_do_not_change_their_buffers():
    op = mx.MxOperand(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), 4, 64)
    with pytest.raises(AttributeError):
        op.codes = torch.zeros(4, 32, dtype=torch.uint8)


def test_an_order_needs_its_slots_without_tokens_too():
    """No tokens, but a capacity above zero: the slots are still written and read."""
    lib, at = mx.load(), 1 << 40
    order = mx.MorExpertOrder(0, 2, 3, 128, 128, 0, at, None, None)
    assert lib.mor_expert_sort(at, C.byref(order), None, 0, None) == 1
    out = mx.MorMxOperand(at, 16, at, 4, 0, 0)
    params = mx.MorMxParams(0, 32, 32, 1, 0, 0, 0, 0)
    assert lib.mor_mx_quantize(C.byref(params), at, C.byref(out), None, C.byref(order), None, None) == 1


# ---- on the GPU --------------------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rule", ["floor", "ceil"])
@pytest.mark.parametrize("tokens, hidden, width", [(1, 32, 40), (7, 100, 33), (130, 256, 300)])
def test_linear(tokens, hidden, width, rule, dtype):
    x, w, dy = made(tokens, hidden, seed=1), made(width, hidden, seed=2, scale=0.1), made(tokens, width, seed=3)
    xg, wg = (t.to(DEV, dtype).requires_grad_() for t in (x, w))
    y = mx_layers.linear(xg, wg, scale_rule=rule, seed=77)
    assert y.dtype == torch.bfloat16
    y.backward(dy.to(DEV))
    assert xg.grad.dtype == dtype and wg.grad.dtype == dtype
    f32 = dtype == torch.float32
    (xq, xt), (wq, wt), (g, gt) = forms(numbers(x), rule), forms(numbers(w), rule), forms(numbers(dy), rule, 77)
    check(y, xq @ wq.T, sums_bound(xq, wq))
    check(xg.grad, g @ wt, sums_bound(g, wt.T), f32)
    check(wg.grad, gt.T @ xt, sums_bound(gt.T, xt.T), f32)


@pytest.mark.gpu
def test_linear_of_one_gradient_or_none_and_strides():
    x, w, dy = made(9, 64, seed=1).to(DEV), made(40, 64, seed=2).to(DEV), made(1, 40, seed=3).to(DEV)
    both = [t.clone().requires_grad_() for t in (x, w)]
    want = mx_layers.linear(*both, seed=5)
    want.backward(dy.expand(9, 40))
    alone = x.clone().requires_grad_()
    mx_layers.linear(alone, w, seed=5).backward(dy.expand(9, 40))           # rows without a stride
    assert torch.equal(alone.grad, both[0].grad)
    alone = w.t().contiguous().t().requires_grad_()                         # columns next to each other
    y = mx_layers.linear(x, alone, seed=5)
    y.backward(dy.expand(9, 40))
    assert torch.equal(alone.grad, both[1].grad) and torch.equal(y, want)
    with torch.no_grad():
        assert torch.equal(mx_layers.linear(*both), want)


LAYERS = [(1, 1, 1, 32, 40), (3, 2, 5, 100, 33), (70, 2, 6, 64, 130), (200, 3, 4, 130, 64)]


def layer(tokens, top_k, experts, hidden, width, seed=0):
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, experts, (tokens, top_k)).astype(np.int32)
    ids[rng.random(ids.shape) < 0.1] = -1
    weights = rng.random((tokens, top_k)).astype(np.float32)
    return (made(tokens, hidden, seed=seed + 1), made(experts, width, hidden, seed=seed + 2, scale=0.1), ids, weights,
            made(tokens, width, seed=seed + 3))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens, top_k, experts, hidden, width", LAYERS)
def test_experts(tokens, top_k, experts, hidden, width, dtype):
    x, w, ids, weights, dy = layer(tokens, top_k, experts, hidden, width)
    xg, wg = (t.to(DEV, dtype).requires_grad_() for t in (x, w))
    weights_g = torch.from_numpy(weights).to(DEV).requires_grad_()
    y = mx_layers.experts(xg, wg, torch.from_numpy(ids).to(DEV), weights_g, seed=9)
    y.backward(dy.to(DEV))

    capacity = mx.expert_capacity(tokens, top_k, experts)
    starts, slot, src = R.sort(ids, experts, 128, capacity)
    used = src >= 0
    rows, grads = np.zeros((capacity, hidden)), np.zeros((capacity, width))
    rows[used] = numbers(x)[src[used] // top_k]
    with np.errstate(over="ignore"):
        grads[used] = (numbers(dy).astype(np.float32)[src[used] // top_k] * weights.reshape(-1)[src[used], None]).astype(np.float64)
    (xq, xt), (g, gt) = forms(rows, "floor"), forms(grads, "floor", 9)
    ys, ys_off, dxs, dxs_off = (np.zeros((capacity, n)) for n in (width, width, hidden, hidden))
    for e in range(experts):
        s = slice(starts[e], starts[e + 1])
        wq, wt = forms(numbers(w[e]), "floor")
        ys[s], ys_off[s] = xq[s] @ wq.T, sums_bound(xq[s], wq)
        dxs[s], dxs_off[s] = g[s] @ wt, sums_bound(g[s], wt.T)
        want = gt[s].T @ xt[s]
        check(wg.grad[e], want, sums_bound(gt[s].T, xt[s].T), dtype == torch.float32)
    ys_off += 2.0 ** -8 * np.abs(ys)
    dxs_off += 2.0 ** -8 * np.abs(dxs)

    def added_up(of, off, factor):
        total, bound = np.zeros((tokens, of.shape[1])), np.zeros((tokens, of.shape[1]))
        for i, at in enumerate(slot):
            if at >= 0:
                total[i // top_k] += factor[i] * of[at]
                bound[i // top_k] += factor[i] * (off[at] + (top_k + 1) * 2.0 ** -24 * np.abs(of[at]))
        return total, bound

    check(y, *added_up(ys, ys_off, weights.reshape(-1).astype(np.float64)))
    check(xg.grad, *added_up(dxs, dxs_off, np.ones(tokens * top_k)))
    dots, dots_off = np.zeros(tokens * top_k), np.zeros(tokens * top_k)
    for i, at in enumerate(slot):
        if at >= 0:
            d = np.abs(numbers(dy)[i // top_k])
            dots[i] = numbers(dy)[i // top_k] @ ys[at]
            dots_off[i] = d @ ys_off[at] + (width + 1) * 2.0 ** -24 * (d @ np.abs(ys[at]))
    check(weights_g.grad, dots.reshape(tokens, top_k), dots_off.reshape(tokens, top_k), True)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens, top_k, experts, hidden, width", LAYERS)
def test_served_experts_answer_as_trained_ones(tokens, top_k, experts, hidden, width):
    x, w, ids, weights, _ = layer(tokens, top_k, experts, hidden, width, seed=20)
    args = x.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(weights).to(DEV)
    with torch.no_grad():
        trained = numbers(mx_layers.experts(args[0], w.to(DEV), *args[1:]))
    served = numbers(mx_layers.ServedExperts(w.to(DEV))(*args))
    # the rows' sums may be in another order, so their BF16 values and the result's may be one unit apart
    xq = R.quantize(numbers(x))[2]
    bound = 2.0 ** -7 * np.abs(trained)
    for j in range(top_k):
        for t in np.nonzero(ids[:, j] >= 0)[0]:
            wq = R.quantize(numbers(w[ids[t, j]]))[2]
            bound[t] += weights[t, j] * (2.0 ** -7 * np.abs(wq @ xq[t]) + 2 * sums_bound(xq[t:t + 1], wq)[0])
    assert (np.abs(trained - served) <= bound).all()


@pytest.mark.gpu
def test_routing_weights_gradient_against_differences():
    """The output is linear in the routing weights up to its roundings: a difference over a step of one is the derivative."""
    tokens, top_k = 20, 2
    x, w, ids, weights, dy = layer(tokens, top_k, 4, 64, 96, seed=40)
    x, w, ids, dy = x.to(DEV), w.to(DEV), torch.from_numpy(ids).to(DEV), dy.to(DEV)
    weights_g = torch.from_numpy(weights).to(DEV).requires_grad_()
    mx_layers.experts(x, w, ids, weights_g).backward(dy)
    with torch.no_grad():
        for j in range(top_k):
            more = weights_g.clone()
            more[:, j] += 1.0
            high, low = (numbers(mx_layers.experts(x, w, ids, v)) for v in (more, weights_g))
            difference = (numbers(dy) * (high - low)).sum(1)
            bound = (np.abs(numbers(dy)) * (np.abs(high) + np.abs(low)) * 2.0 ** -8).sum(1) + 1e-6
            assert (np.abs(difference - numbers(weights_g.grad)[:, j]) <= bound).all()


@pytest.mark.gpu
def test_training_learns():
    losses = mx_layers.train()
    assert np.isfinite(losses).all() and np.mean(losses[-5:]) < 0.6 * np.mean(losses[:2])


@pytest.mark.gpu
def test_wrong_inputs_raise():
    x, w, ids, weights, _ = layer(4, 2, 3, 64, 40)
    x, w, ids, weights = x.to(DEV), w.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(weights).to(DEV)
    with pytest.raises(ValueError):
        mx_layers.experts(x, w, ids.long(), weights)
    with pytest.raises(ValueError):
        mx_layers.experts(x, w, ids, weights[:3])
    with pytest.raises(ValueError):
        mx_layers.ServedExperts(w)(x[:, :32], ids, weights)
    with pytest.raises(binding.MorError):
        mx.mor_mx_quantize(x[:1].expand(4, 64), mx.alloc_operand(4, 64, DEV))       # rows upon each other


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_tokens(dtype):
    w = made(40, 64, seed=2).to(DEV, dtype).requires_grad_()
    x = torch.empty(0, 64, device=DEV, dtype=dtype).requires_grad_()
    y = mx_layers.linear(x, w)
    y.backward(torch.empty_like(y))
    assert y.shape == (0, 40) and x.grad.shape == (0, 64) and (w.grad == 0).all()
    w = made(3, 40, 64, seed=2).to(DEV, dtype).requires_grad_()
    ids, weights = torch.empty(0, 2, device=DEV, dtype=torch.int32), torch.empty(0, 2, device=DEV).requires_grad_()
    y = mx_layers.experts(x, w, ids, weights)
    y.backward(torch.empty_like(y))
    assert y.shape == (0, 40) and (w.grad == 0).all() and weights.grad.shape == (0, 2)
    assert mx_layers.ServedExperts(w)(x, ids, weights.detach()).shape == (0, 40)


@pytest.mark.gpu
def test_every_choice_dropped():
    x, w, ids, weights, dy = layer(5, 2, 3, 64, 40)
    x, w = x.to(DEV).requires_grad_(), w.to(DEV).requires_grad_()
    weights = torch.from_numpy(weights).to(DEV).requires_grad_()
    y = mx_layers.experts(x, w, torch.full((5, 2), -1, device=DEV, dtype=torch.int32), weights)
    y.backward(dy.to(DEV))
    for t in (y, x.grad, w.grad, weights.grad):
        assert (t == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2])
def test_experts_of_one_gradient(which):
    x, w, ids, weights, dy = layer(50, 2, 4, 96, 72, seed=60)
    ids, dy = torch.from_numpy(ids).to(DEV), dy.to(DEV)
    every = [t.to(DEV).requires_grad_() for t in (x, w, torch.from_numpy(weights))]
    mx_layers.experts(every[0], every[1], ids, every[2], seed=4).backward(dy)
    one = [t.detach().clone().requires_grad_(i == which) for i, t in enumerate(every)]
    mx_layers.experts(one[0], one[1], ids, one[2], seed=4).backward(dy)
    assert torch.equal(one[which].grad, every[which].grad)


@pytest.mark.gpu
def test_layers_in_a_graph():
    """Captured once, replayed on other inputs, with eager work in between."""
    x, w, ids, weights, _ = layer(70, 2, 6, 64, 130, seed=80)
    served, x, ids, weights = mx_layers.ServedExperts(w.to(DEV)), x.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(weights).to(DEV)
    with torch.cuda.stream(torch.cuda.Stream()):
        served(x, ids, weights)                                             # (allocations before the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = served(x, ids, weights)
    for step in range(4):
        x.copy_(made(70, 64, seed=90 + step))
        ids.copy_(torch.randint(-1, 6, (70, 2), generator=torch.Generator().manual_seed(step), dtype=torch.int32))
        want = served(x, ids, weights)
        torch.cuda.synchronize()
        y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
