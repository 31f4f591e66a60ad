"""What a training step asks of the layers beyond their products: rounding without bias, fresh random bits, second derivatives that are
refused instead of lost, operands kept where autograd sees them, no work that nothing reads, gradients in the bits of their type."""
import numpy as np
import pytest
import torch

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
