"""Which device and stream a call of the 4-bit operators goes to, without a GPU: tensors that say they live on one, and a library that
only notes its calls.  Tensors on several devices, or some in host memory, are refused before the library is called; those on a
device that is not the current one are launched there."""
import contextlib

import pytest
import torch

from paper_2512_22804_amd import binding, mx


class On:
    """A host tensor that says it lives on device `index`."""

    def __init__(self, t, index):
        self._t, self._index = t, index
        self.is_cuda, self.device = index >= 0, torch.device("cuda", index) if index >= 0 else torch.device("cpu")

    def get_device(self):
        return self._index

    def __getattr__(self, name):
        return getattr(self._t, name)


class Library:
    def __init__(self, calls, current):
        self.calls, self.current = calls, current

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.current[-1], args[-1]))
            return 0
        return call


@pytest.fixture
def calls(monkeypatch):
    """(function, current device, stream) of every call; streams are called 100 + their device."""
    made, current = [], [0]

    @contextlib.contextmanager
    def device(index):
        current.append(index)
        yield
        current.pop()

    mx.load()
    monkeypatch.setattr(mx, "_lib", Library(made, current))
    monkeypatch.setattr(binding, "_raw_stream", lambda index: 100 + index)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[-1])
    monkeypatch.setattr(torch.cuda, "device", device)
    return made


T, K, D, N, E, CAP = 4, 2, 64, 96, 3, 512


def bf16(rows, cols, index):
    return On(torch.zeros(rows, cols, dtype=torch.bfloat16), index)


def f32(n, index):
    return On(torch.zeros(n), index)


def ints(n, index):
    return On(torch.zeros(n, dtype=torch.int32), index)


def operand(rows, cols, index, batch=None):
    lead = (rows,) if batch is None else (batch, rows)
    return mx.MxOperand(On(torch.zeros(*lead, cols // 2, dtype=torch.uint8), index), On(torch.zeros(*lead, 4 * -(-cols // 128), dtype=torch.uint8), index),
                        rows, cols)


def order(index, workspace=None):
    return mx.ExpertOrder(T, K, E, 128, CAP, ints(E + 1, index), ints(T * K, index), ints(CAP, index), workspace)


# every call and the things that it takes, each on a device of its own
CALLS = {
    "mor_mx_quantize": (mx.mor_mx_quantize, [lambda i: bf16(T, D, i), lambda i: operand(CAP, D, i), lambda i: operand(D, CAP, i), lambda i: order(i),
                                             lambda i: f32(T * K, i)], lambda f, x, o, ot, r, w: f(x, o, ot, order=r, weights=w)),
    "mor_mx_dequantize": (mx.mor_mx_dequantize, [lambda i: operand(T, D, i), lambda i: bf16(T, D, i)], lambda f, *a: f(*a)),
    "mor_mx_product": (mx.mor_mx_product, [lambda i: operand(T, D, i), lambda i: operand(N, D, i), lambda i: bf16(T, N, i),
                                           lambda i: On(torch.zeros(8, dtype=torch.uint8), i)], lambda f, *a: f(*a)),
    "mor_mx_product_rows": (mx.mor_mx_product_rows, [lambda i: operand(CAP, D, i), lambda i: operand(N, D, i, E), lambda i: order(i),
                                                     lambda i: bf16(CAP, N, i)], lambda f, *a: f(*a)),
    "mor_mx_product_depth": (mx.mor_mx_product_depth, [lambda i: operand(D, CAP, i), lambda i: operand(N, CAP, i), lambda i: order(i),
                                                       lambda i: On(torch.zeros(E, D, N), i)], lambda f, *a: f(*a)),
    "mor_expert_sort": (mx.mor_expert_sort, [lambda i: ints(T * K, i), lambda i: order(i)], lambda f, *a: f(*a)),
    "mor_expert_gather": (mx.mor_expert_gather, [lambda i: bf16(T, D, i), lambda i: order(i), lambda i: bf16(CAP, D, i)], lambda f, *a: f(*a)),
    "mor_expert_combine": (mx.mor_expert_combine, [lambda i: bf16(CAP, D, i), lambda i: order(i), lambda i: f32(T * K, i), lambda i: bf16(T, D, i)],
                           lambda f, *a: f(*a)),
    "mor_expert_combine_backward": (mx.mor_expert_combine_backward, [lambda i: bf16(T, D, i), lambda i: bf16(CAP, D, i), lambda i: order(i),
                                                                     lambda i: f32(T * K, i), lambda i: bf16(CAP, D, i), lambda i: f32(T * K, i)],
                                    lambda f, *a: f(*a)),
}


@pytest.mark.parametrize("index", [0, 1])
@pytest.mark.parametrize("name", CALLS)
def test_launched_where_the_tensors_are(calls, name, index):
    function, things, call = CALLS[name]
    call(function, *[make(index) for make in things])
    assert calls == [(name, index, 100 + index)]


@pytest.mark.parametrize("name", CALLS)
def test_several_devices_are_refused(calls, name):
    function, things, call = CALLS[name]
    for odd in range(len(things)):
        for index in (1, -1):               # another device, host memory
            with pytest.raises(ValueError):
                call(function, *[make(index if at == odd else 0) for at, make in enumerate(things)])
    assert not calls


def test_operands_and_orders_of_several_devices_are_refused(calls):
    codes, scales = On(torch.zeros(4, 32, dtype=torch.uint8), 0), On(torch.zeros(4, 4, dtype=torch.uint8), 1)
    with pytest.raises(ValueError):
        mx.MxOperand(codes, scales, 4, 64)
    for odd in range(4):
        at = [1 if odd == i else 0 for i in range(4)]
        with pytest.raises(ValueError):
            mx.ExpertOrder(T, K, E, 128, CAP, ints(E + 1, at[0]), ints(T * K, at[1]), ints(CAP, at[2]), On(torch.zeros(8, dtype=torch.uint8), at[3]))
