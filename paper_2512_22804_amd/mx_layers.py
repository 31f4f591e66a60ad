"""The microscaled 4-bit operators as a model uses them: a linear layer and a layer of experts, with their gradients for training and
their form without for serving.  ``python -m paper_2512_22804_amd.mx_layers`` trains both on made-up data and serves the result.

Every product reads 4-bit operands whose blocks lie along its depth, so an operand of a training step is quantised in two forms from
one read: as it is and transposed.  Activations and weights are rounded to nearest, gradients stochastically, whose errors
average out over steps, if nothing is clipped: under the floor rule magnitudes in (6, 8) times a block's scale become 6 times it
whatever the random bits (the mean over draws of normal numbers is off by 4 % of their norm), under the ceil rule none does.  What is quantised in the
forward pass for the backward pass is kept in 4 bits, not in 16.
"""
from __future__ import annotations

import functools

import torch

from . import mx


def _bf16(t: torch.Tensor) -> torch.Tensor:
    """What is quantised.  Float32 values are rounded to BF16 before they are rounded to four bits, by a pass of torch's: off by 2^-9 of
    themselves before a step of 2^-3."""
    t = t.detach().to(torch.bfloat16)
    return t if t.stride(-1) == 1 and t.stride(-2) >= t.shape[-1] else t.contiguous()


def _check(x: torch.Tensor, w: torch.Tensor, dims: int) -> None:
    for t, name in ((x, "x"), (w, "w")):
        if t.dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"{name}: {t.dtype} is neither torch.bfloat16 nor torch.float32")
    if x.dim() != 2 or w.dim() != dims or x.shape[-1] != w.shape[-1]:
        raise ValueError(f"shapes do not match: x {tuple(x.shape)}, w {tuple(w.shape)}")


def _check_choices(x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor) -> None:
    # (weights one after the other, in the choices' order, are as good; of another shape they would be another choice's)
    if ids.dim() != 2 or ids.shape[0] != x.shape[0] or weights.shape not in (ids.shape, (ids.numel(),)):
        raise ValueError(f"shapes do not match: x {tuple(x.shape)}, ids {tuple(ids.shape)}, weights {tuple(weights.shape)}")


def _gradients(scale_rule: str, seed: int | None, gradient_rule: str | None, rounds: bool) -> dict:
    """How a call's gradients are rounded.  Without a seed of the caller's it is a new one, if there is a gradient to round at all."""
    if gradient_rule is None:
        gradient_rule = "ceil" if seed is None else scale_rule
    for rule in (scale_rule, gradient_rule):
        if rule not in mx.SCALE_RULE:
            raise ValueError(f"{rule!r} is not one of {tuple(mx.SCALE_RULE)}")
    if seed is None:
        seed = int(torch.randint(1 << 62, ())) if rounds else 0
    return dict(scale_rule=gradient_rule, rounding="stochastic", seed=seed)


def _product(a: mx.MxOperand, b: mx.MxOperand, dtype: torch.dtype) -> torch.Tensor:
    if a.cols == 0:                     # no tokens: a gradient without terms
        return torch.zeros(a.rows, b.rows, dtype=dtype, device=a.codes.device)
    c = torch.empty(a.rows, b.rows, dtype=dtype, device=a.codes.device)
    mx.mor_mx_product(a, b, c, mx.alloc_product_workspace(a, b, c.device))
    return c


def _operands(x: torch.Tensor, rows: int, cols: int, transposed: bool = True, batch: int | None = None, plain: bool = True, **how):
    """``x`` as an operand of ``rows`` x ``cols`` and its transpose, None for what is not wanted."""
    out = mx.alloc_operand(rows, cols, x.device, batch) if plain else None
    out_t = mx.alloc_operand(cols, rows, x.device, batch) if transposed else None
    mx.mor_mx_quantize(x, out, out_t, **how)
    return out, out_t


def _saved(operand: mx.MxOperand | None) -> tuple:
    """An operand as tensors for autograd to keep: hooks on saved tensors see them, and they go with the graph's buffers."""
    return (None, None) if operand is None else (operand.codes, operand.scales)


def _restored(codes: torch.Tensor | None, scales: torch.Tensor | None, rows: int, cols: int) -> mx.MxOperand | None:
    return None if codes is None else mx.MxOperand(codes, scales, rows, cols)


class _NoFurther(torch.autograd.Function):
    """Gradients as they are, whose own derivatives raise.  ``anchor`` requires a gradient, so that they do."""

    @staticmethod
    def forward(ctx, anchor, *grads):
        return tuple(g.view_as(g) for g in grads)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the 4-bit layers have first derivatives only: their gradients cannot be differentiated again")


def _first_derivatives(backward):
    """The kernels record no graph, so with ``create_graph`` the gradients' dependence on the inputs would be lost silently, also where ``dy``
    does not depend on them."""
    @functools.wraps(backward)
    def wrapped(ctx, dy):
        with torch.no_grad():
            grads = backward(ctx, dy)
        if torch.is_grad_enabled():
            there = [g for g in grads if g is not None]
            there = iter(_NoFurther.apply(torch.empty(0, requires_grad=True), *there))
            grads = tuple(None if g is None else next(there) for g in grads)
        return grads
    return wrapped


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, scale_rule, how, training):
        tokens, hidden = x.shape
        # either input's transpose is what the other one's gradient reads
        xq, xt = _operands(_bf16(x), tokens, hidden, training and ctx.needs_input_grad[1], scale_rule=scale_rule)
        wq, wt = _operands(_bf16(w), w.shape[0], hidden, training and ctx.needs_input_grad[0], scale_rule=scale_rule)
        ctx.save_for_backward(*_saved(xt), *_saved(wt))
        ctx.sizes, ctx.how, ctx.types = (tokens, hidden, w.shape[0]), how, (x.dtype, w.dtype)
        return _product(xq, wq, torch.bfloat16)

    @staticmethod
    @_first_derivatives
    def backward(ctx, dy):
        tokens, hidden, width = ctx.sizes
        kept = ctx.saved_tensors
        xt, wt = _restored(*kept[:2], hidden, tokens), _restored(*kept[2:], hidden, width)
        g, gt = _operands(_bf16(dy), dy.shape[0], dy.shape[1], xt is not None, plain=wt is not None, **ctx.how)
        dx = _product(g, wt, ctx.types[0]) if wt is not None else None
        dw = _product(gt, xt, ctx.types[1]) if xt is not None else None
        return dx, dw, None, None, None


def linear(x: torch.Tensor, w: torch.Tensor, scale_rule: str = "floor", seed: int | None = None, gradient_rule: str | None = None) -> torch.Tensor:
    """``x`` (tokens, hidden) times ``w`` (width, hidden), transposed, in BF16.  ``x`` and ``w`` are BF16 or float32, which their gradients then
    are too.

    ``seed``: of the gradients' rounding, another one each step and layer; None: every call draws one from torch's generator on
    the host (a captured graph repeats the one that was drawn).  ``gradient_rule``: the scale rule of the gradients, "ceil" for rounding
    without bias, which is what a call without a seed does; with a seed it is ``scale_rule`` unless given, so that such
    calls repeat what they have always answered."""
    _check(x, w, 2)
    training = torch.is_grad_enabled()
    how = _gradients(scale_rule, seed, gradient_rule, training and (x.requires_grad or w.requires_grad))
    return _Linear.apply(x, w, scale_rule, how, training)


def _row_type(x: torch.Tensor) -> torch.dtype:
    """Of the experts' rows between the product and the sum over a token's choices, and of the tokens' gradient: BF16 where the tokens are,
    one rounding more for half of the bytes; float32, without it, where those are float32."""
    return torch.float32 if x.dtype == torch.float32 else torch.bfloat16


class _Experts(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, ids, weights, scale_rule, how, training):
        tokens, hidden = x.shape
        experts, width = w.shape[:2]
        # segments of whole 128 rows: the matrices' gradients are sums over them
        order = mx.alloc_order(tokens, ids.shape[1], experts, x.device, align=128)
        mx.mor_expert_sort(ids, order)
        xq, xt = _operands(_bf16(x), order.capacity, hidden, training and ctx.needs_input_grad[1], scale_rule=scale_rule, order=order)
        wq, wt = _operands(_bf16(w), width, hidden, training and ctx.needs_input_grad[0], experts, scale_rule=scale_rule)
        ys = torch.empty(order.capacity, width, dtype=_row_type(x), device=x.device)
        mx.mor_mx_product_rows(xq, wq, order, ys)
        y = torch.empty(tokens, width, dtype=torch.bfloat16, device=x.device)
        weights = weights.detach().contiguous()
        mx.mor_expert_combine(ys, order, weights, y)
        ctx.save_for_backward(weights, order.offsets, order.slot_of, order.src, ys if ctx.needs_input_grad[3] else None, *_saved(xt), *_saved(wt))
        ctx.sizes = (order.tokens, order.top_k, order.n_experts, order.align, order.capacity), hidden, width
        ctx.how, ctx.types = how, (x.dtype, w.dtype)
        return y

    @staticmethod
    @_first_derivatives
    def backward(ctx, dy):
        sizes, hidden, width = ctx.sizes
        weights, offsets, slot_of, src, ys, *kept = ctx.saved_tensors
        order = mx.ExpertOrder(*sizes, offsets, slot_of, src, None)
        xt, wt = _restored(*kept[:2], hidden, order.capacity), _restored(*kept[2:], hidden, width)
        dy = _bf16(dy)
        dx = dw = dweights = None
        if xt is not None or wt is not None:
            # the rows' gradients, each times its choice's weight, go from the tokens' straight into 4 bits
            g, gt = _operands(dy, order.capacity, dy.shape[1], xt is not None, plain=wt is not None, order=order, weights=weights, **ctx.how)
        if wt is not None:
            dxs = torch.empty(order.capacity, wt.rows, dtype=ctx.types[0], device=dy.device)
            mx.mor_mx_product_rows(g, wt, order, dxs)
            dx = torch.empty(order.tokens, wt.rows, dtype=ctx.types[0], device=dy.device)
            mx.mor_expert_combine(dxs, order, None, dx)
        if xt is not None:
            dw = torch.empty(order.n_experts, dy.shape[1], xt.rows, dtype=ctx.types[1], device=dy.device)
            mx.mor_mx_product_depth(gt, xt, order, dw)
        if ctx.needs_input_grad[3]:
            dweights = torch.empty_like(weights)
            mx.mor_expert_combine_backward(dy, ys, order, None, None, dweights)
        return dx, dw, None, dweights, None, None, None


def experts(x: torch.Tensor, w: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor, scale_rule: str = "floor",
            seed: int | None = None, gradient_rule: str | None = None) -> torch.Tensor:
    """Sum over a token's choices ``ids`` (tokens, top_k; int32, outside the experts: dropped) of its ``weights`` (tokens, top_k; float32) times
    the token's row of ``x`` (tokens, hidden) times that expert's matrix of ``w`` (experts, width, hidden), transposed; in BF16.  Float32
    tokens keep the experts' rows in float32 until they are added up, and get a float32 gradient.  ``seed`` and
    ``gradient_rule`` as for :func:`linear`."""
    _check(x, w, 3)
    _check_choices(x, ids, weights)
    training = torch.is_grad_enabled()
    how = _gradients(scale_rule, seed, gradient_rule, training and (x.requires_grad or w.requires_grad))
    return _Experts.apply(x, w, ids.contiguous(), weights, scale_rule, how, training)


class ServedExperts:
    """The experts' matrices in 4 bits, for tokens as they come: no gradient, segments as short as the tokens make them."""

    def __init__(self, w: torch.Tensor, scale_rule: str = "floor"):
        if w.dim() != 3:
            raise ValueError(f"w must be (experts, width, hidden), not {tuple(w.shape)}")
        self.scale_rule = scale_rule
        self.w, _ = _operands(_bf16(w), w.shape[1], w.shape[2], False, w.shape[0], scale_rule=scale_rule)

    def __call__(self, x: torch.Tensor, ids: torch.Tensor, weights: torch.Tensor) -> torch.Tensor:
        if x.dim() != 2 or x.shape[1] != self.w.cols:
            raise ValueError(f"x must be (tokens, {self.w.cols}), not {tuple(x.shape)}")
        _check_choices(x, ids, weights)
        tokens, hidden = x.shape
        order = mx.alloc_order(tokens, ids.shape[1], self.w.batch, x.device, align=1)
        mx.mor_expert_sort(ids.contiguous(), order)
        xq, _ = _operands(_bf16(x), order.capacity, hidden, False, scale_rule=self.scale_rule, order=order)
        ys = torch.empty(order.capacity, self.w.rows, dtype=_row_type(x), device=x.device)
        mx.mor_mx_product_rows(xq, self.w, order, ys)
        y = torch.empty(tokens, self.w.rows, dtype=torch.bfloat16, device=x.device)
        mx.mor_expert_combine(ys, order, weights.contiguous(), y)
        return y


def train(steps: int = 60, tokens: int = 512, hidden: int = 256, width: int = 192, n_experts: int = 8, top_k: int = 2, device="cuda") -> list[float]:
    """A linear layer, a router's choice and a layer of experts learn what such layers with other weights answer; the losses."""
    made = torch.Generator(device=device).manual_seed(0)
    normal = lambda *shape: torch.randn(*shape, generator=made, device=device)
    shapes = ((hidden, hidden), (n_experts, width, hidden), (n_experts, hidden))
    goal = [normal(*s) * hidden ** -0.5 for s in shapes]
    mine = [(g + 0.5 * hidden ** -0.5 * normal(*s)).requires_grad_() for g, s in zip(goal, shapes)]
    optimizer = torch.optim.Adam(mine, lr=2e-3)

    def answer(x, params, ids, seed):
        h = linear(x, params[0], seed=seed, gradient_rule="ceil")
        chosen = (x.float() @ params[2].t()).gather(1, ids.long()).softmax(dim=1)
        return experts(h, params[1], ids, chosen, seed=seed + 1, gradient_rule="ceil")

    losses = []
    for step in range(steps):
        x = normal(tokens, hidden).to(torch.bfloat16)
        ids = (x.float() @ goal[2].t()).topk(top_k, dim=1).indices.to(torch.int32)
        with torch.no_grad():
            wanted = answer(x, goal, ids, 0)
        loss = (answer(x, mine, ids, 2 * step + 1).float() - wanted.float()).square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
    return losses


def main() -> None:
    losses = train()
    print("loss of every tenth step: " + ", ".join(f"{v:.4f}" for v in losses[::10] + losses[-1:]))
    torch.manual_seed(0)
    served = ServedExperts(torch.randn(8, 192, 256, device="cuda") / 16)
    x = torch.randn(3, 256, device="cuda").to(torch.bfloat16)
    ids = torch.randint(0, 8, (3, 2), device="cuda", dtype=torch.int32)
    y = served(x, ids, torch.full((3, 2), 0.5, device="cuda"))
    print(f"three tokens served: {tuple(y.shape)}, of mean square {y.float().square().mean().item():.3f}")


if __name__ == "__main__":
    main()
