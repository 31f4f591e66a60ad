"""What a training step asks of the layers beyond their products: rounding without bias, fresh random bits, second derivatives that are
refused instead of lost, operands kept where autograd sees them, no work that nothing reads, gradients in the bits of their type."""
import numpy as np
import pytest
import torch
import torch.utils.checkpoint

import mx_refmodel as R
from paper_2512_22804_amd import mx, mx_layers
from test_mx_layers import check, forms, layer, numbers, sums_bound

pytestmark = pytest.mark.gpu
DEV = "cuda"


def answer(kind, x, w, args, **how):
    return mx_layers.linear(x, w, **how) if kind == "linear" else mx_layers.experts(x, w, *args, **how)


def gradients(kind, dy, x, w, args, **how):
    """Gradients of the tokens and of the weights."""
    x, w = x.clone().requires_grad_(), w.clone().requires_grad_()
    answer(kind, x, w, args, **how).backward(dy)
    return x.grad, w.grad


def case(kind, tokens=128, hidden=96, width=64):
    """Tokens and weights that four bits hold exactly, gradients of which every other row's largest elements are 7: under the floor rule
    those become 6, whatever the random bits.  With the layer's gradients in binary64."""
    grid = torch.tensor([-2.0, -1.0, 0.0, 1.0, 2.0, 4.0])
    draw = lambda seed, *s: grid[torch.randint(0, 6, s, generator=torch.Generator().manual_seed(seed))].to(DEV)
    x, dy = draw(1, tokens, hidden), draw(3, tokens, width)
    dy[::2] = dy[::2] * 0.8125 + 3.75               # 2.125 .. 7, all exact in BF16
    dy = dy.to(torch.bfloat16)
    if kind == "linear":
        w, args = draw(2, width, hidden), ()
        matrices, mine = [w], [slice(None)]
    else:
        w = draw(2, 2, width, hidden)
        args = ((torch.arange(tokens, device=DEV) % 2).to(torch.int32)[:, None], torch.ones(tokens, 1, device=DEV))
        matrices, mine = list(w), [slice(0, None, 2), slice(1, None, 2)]
    return x, w, args, dy, matrices, mine


@pytest.mark.parametrize("kind", ["linear", "experts"])
def test_random_bits(kind):
    """A call without a seed draws one, from torch's generator on the host and only if there is a gradient to round; a seed fixes the bits."""
    x, w, args, dy, *_ = case(kind)
    torch.manual_seed(5)
    first, second = gradients(kind, dy, x, w, args), gradients(kind, dy, x, w, args)
    torch.manual_seed(5)
    again = gradients(kind, dy, x, w, args)
    for a, b, c in zip(first, second, again):
        assert not torch.equal(a, b) and torch.equal(a, c)
    for a, b in zip(gradients(kind, dy, x, w, args, seed=9), gradients(kind, dy, x, w, args, seed=9)):
        assert torch.equal(a, b)
    before = torch.get_rng_state()
    answer(kind, x, w, args)
    with torch.no_grad():
        answer(kind, x.clone().requires_grad_(), w, args)
    assert torch.equal(before, torch.get_rng_state())


@pytest.mark.parametrize("how", [{}, {"gradient_rule": "ceil", "seed": 1}])
@pytest.mark.parametrize("kind", ["linear", "experts"])
def test_gradients_have_no_bias(kind, how):
    """Every rounding error E of dy has a step of 2 at most (scale 2, magnitudes below 8), so a mean of zero and a variance of 1 at most.  The
    mean gradient of n calls, less the exact one, is E w (or E^T x) with E's variances divided by n; its scalar product with a
    gradient G is that of E and G w^T (x G^T): of standard deviation |G w^T| / sqrt(n) at most.  Six of those, and 2^-8 of |G|^2
    for roundings to BF16.  (A clipped 7 is off by 1 in every call: 2 to 4 % of |G|^2.)"""
    x, w, args, dy, matrices, mine = case(kind)
    n = 64
    total_x, total_w = torch.zeros(x.shape, device=DEV, dtype=torch.float64), torch.zeros(w.shape, device=DEV, dtype=torch.float64)
    for i in range(n):
        if "seed" in how:
            how = dict(how, seed=how["seed"] + 1)
        gx, gw = gradients(kind, dy, x, w, args, **how)
        total_x += gx.double()
        total_w += gw.double()
    total_w = [total_w] if kind == "linear" else list(total_w)
    for matrix, rows, got_w in zip(matrices, mine, total_w):
        a, b, m = x[rows].double(), dy[rows].double(), matrix.double()
        for got, want, spread in ((total_x[rows], b @ m, (b @ m) @ m.t()), (got_w, b.t() @ a, a @ (b.t() @ a).t())):
            off = float(((got / n - want) * want).sum())
            assert abs(off) <= 6 * float(spread.norm()) / n ** 0.5 + 2.0 ** -8 * float((want * want).sum()), off / float((want * want).sum())


@pytest.mark.parametrize("kind", ["linear", "experts"])
def test_gradient_rule(kind):
    """The gradients' scale rule alone; without one a call with a seed follows the other operands' rule."""
    x, w, args, dy, *_ = case(kind)
    how = {rule: gradients(kind, dy, x, w, args, seed=3, gradient_rule=rule) for rule in ("floor", "ceil")}
    for a, b, c in zip(how["floor"], gradients(kind, dy, x, w, args, seed=3), how["ceil"]):
        assert torch.equal(a, b) and not torch.equal(a, c)
    with pytest.raises(ValueError):
        answer(kind, x, w, args, gradient_rule="round")


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("kind", ["linear", "experts"])
def test_second_derivatives_raise(kind, which):
    x, w, args, dy, *_ = case(kind)
    inputs = [x, w, *args[1:]]
    if which >= len(inputs):
        which = 0
    inputs = [t.clone().requires_grad_() for t in inputs]
    y = answer(kind, inputs[0], inputs[1], (*args[:1], *inputs[2:]), seed=3)
    loss = (y.float() * dy.float()).sum()
    first, = torch.autograd.grad(loss, inputs[which], retain_graph=True)
    g, = torch.autograd.grad(loss, inputs[which], create_graph=True)
    assert torch.equal(g, first) and not first.requires_grad
    with pytest.raises(RuntimeError):
        (loss + g.square().sum()).backward()        # (without the loss there is nothing to differentiate, which raises too)


@pytest.mark.parametrize("kind", ["linear", "experts"])
def test_kept_operands_are_saved_tensors(kind):
    """Hooks on saved tensors see the operands that the backward pass reads, may keep them elsewhere, and the graph lets go of them."""
    x, w, args, dy, *_ = case(kind)
    want = gradients(kind, dy, x, w, args, seed=3)
    sizes = []

    def pack(t):
        sizes.append(t.numel() * t.element_size())
        return t.cpu()

    a, b = x.clone().requires_grad_(), w.clone().requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t.to(DEV)):
        y = answer(kind, a, b, args, seed=3)
    assert sum(sizes) >= (x.numel() + w.numel()) * 17 // 32                     # both transposes
    y.backward(dy, retain_graph=True)
    assert torch.equal(a.grad, want[0]) and torch.equal(b.grad, want[1])
    y.backward(dy)
    assert torch.equal(a.grad, 2 * want[0]) and torch.equal(b.grad, 2 * want[1])
    with pytest.raises(RuntimeError):
        y.backward(dy)


@pytest.mark.parametrize("reentrant", [False, True])
@pytest.mark.parametrize("kind", ["linear", "experts"])
def test_checkpointing(kind, reentrant):
    x, w, args, dy, *_ = case(kind)
    torch.manual_seed(6)
    want = gradients(kind, dy, x, w, args)
    torch.manual_seed(6)
    a, b = x.clone().requires_grad_(), w.clone().requires_grad_()
    torch.utils.checkpoint.checkpoint(lambda a, b: answer(kind, a, b, args), a, b, use_reentrant=reentrant).backward(dy)
    assert torch.equal(a.grad, want[0]) and torch.equal(b.grad, want[1])


@pytest.mark.parametrize("kind", ["linear", "experts"])
def test_inference_mode(kind):
    x, w, args, *_ = case(kind)
    want = answer(kind, x, w, args)
    with torch.inference_mode():
        assert torch.equal(answer(kind, x.clone().requires_grad_(), w, args), want)


@pytest.mark.parametrize("kind", ["linear", "experts"])
def test_forms_that_nothing_reads_are_not_made(kind, monkeypatch):
    """dy as it is for the tokens' gradient, transposed for the weights', and nothing for the routing weights' alone."""
    x, w, args, dy, *_ = case(kind)
    made = []
    quantize = mx.mor_mx_quantize

    def note(x, out=None, out_t=None, **how):
        made.append((out is not None, out_t is not None))
        quantize(x, out, out_t, **how)

    for need_x, need_w in ((True, True), (True, False), (False, True), (False, False)):
        a, b = x.clone().requires_grad_(need_x), w.clone().requires_grad_(need_w)
        router = [t.clone().requires_grad_() if t.is_floating_point() else t for t in args]
        y = answer(kind, a, b, router, seed=3)
        if y.requires_grad:
            with monkeypatch.context() as m:
                m.setattr(mx, "mor_mx_quantize", note)
                made.clear()
                y.backward(dy)
            assert made == ([(need_x, need_w)] if need_x or need_w else [])


def test_experts_of_binary32_tokens_keep_binary32_rows():
    """Rows between product and sum, the tokens' gradient and the routing weights' gradient without a rounding to BF16: each element is within
    the products' bounds, the sums' (top_k + 1) 2^-24 or d 2^-24, and one rounding to the type of the result.  Routing weights of both
    signs, so that rows cancel."""
    tokens, top_k, experts, hidden, width = 150, 3, 4, 130, 64
    x, w, ids, weights, dy = layer(tokens, top_k, experts, hidden, width, seed=7)
    weights = np.where(np.arange(top_k) % 2, -weights, weights).astype(np.float32)
    xg, wg = (t.to(DEV, torch.float32).requires_grad_() for t in (x, w))
    weights_g = torch.from_numpy(weights).to(DEV).requires_grad_()
    y = mx_layers.experts(xg, wg, torch.from_numpy(ids).to(DEV), weights_g, seed=9)
    y.backward(dy.to(DEV))
    served = mx_layers.ServedExperts(w.to(DEV))(x.to(DEV, torch.float32), torch.from_numpy(ids).to(DEV), torch.from_numpy(weights).to(DEV))

    capacity = mx.expert_capacity(tokens, top_k, experts)
    starts, slot, src = R.sort(ids, experts, 128, capacity)
    used = src >= 0
    rows, grads = np.zeros((capacity, hidden)), np.zeros((capacity, width))
    rows[used] = numbers(x)[src[used] // top_k]
    grads[used] = (numbers(dy).astype(np.float32)[src[used] // top_k] * weights.reshape(-1)[src[used], None]).astype(np.float64)
    xq, g = forms(rows, "floor")[0], forms(grads, "floor", 9)[0]
    ys, ys_off, dxs, dxs_off = (np.zeros((capacity, n)) for n in (width, width, hidden, hidden))
    for e in range(experts):
        s = slice(starts[e], starts[e + 1])
        wq, wt = forms(numbers(w[e]), "floor")
        ys[s], ys_off[s] = xq[s] @ wq.T, sums_bound(xq[s], wq)
        dxs[s], dxs_off[s] = g[s] @ wt, sums_bound(g[s], wt.T)
    ys_off += 2.0 ** -24 * np.abs(ys)
    dxs_off += 2.0 ** -24 * np.abs(dxs)

    def added_up(of, off, factor):
        total, bound = np.zeros((tokens, of.shape[1])), np.zeros((tokens, of.shape[1]))
        for i, at in enumerate(slot):
            if at >= 0:
                total[i // top_k] += factor[i] * of[at]
                bound[i // top_k] += abs(factor[i]) * (off[at] + (top_k + 1) * 2.0 ** -24 * np.abs(of[at]))
        return total, bound

    for got in (y, served):
        check(got, *added_up(ys, ys_off, weights.reshape(-1).astype(np.float64)))
    check(xg.grad, *added_up(dxs, dxs_off, np.ones(tokens * top_k)), True)
    dots, dots_off = np.zeros(tokens * top_k), np.zeros(tokens * top_k)
    for i, at in enumerate(slot):
        if at >= 0:
            d = np.abs(numbers(dy)[i // top_k])
            dots[i] = numbers(dy)[i // top_k] @ ys[at]
            dots_off[i] = d @ ys_off[at] + (width + 1) * 2.0 ** -24 * (d @ np.abs(ys[at]))
    check(weights_g.grad, dots.reshape(tokens, top_k), dots_off.reshape(tokens, top_k), True)
