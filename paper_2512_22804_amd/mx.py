"""Thin ctypes binding of the microscaled 4-bit operands, their products and the sorting of tokens by expert (the C ABI
declared in ``include/mor_mx.h``, exported by ``libmor.so``).

Argument marshalling only, as in :mod:`binding`: tensors are checked for what the C ABI cannot see (device, type, shape,
strides), and every call raises :class:`binding.MorError` for what it refuses.  What a call takes lives on one device; it is enqueued on
that device's current stream.
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

import torch

from . import binding

BLOCK = 32
SCALE_RULE = {"floor": 0, "ceil": 1}
ROUNDING = {"nearest": 0, "stochastic": 1}
EXPERTS_MAX = 1024

EXPORTS = ("mor_mx_quantize", "mor_mx_dequantize", "mor_mx_product_workspace_bytes", "mor_mx_product", "mor_mx_product_rows",
           "mor_mx_product_depth", "mor_expert_capacity", "mor_expert_workspace_bytes", "mor_expert_sort", "mor_expert_gather",
           "mor_expert_combine", "mor_expert_combine_f32", "mor_expert_combine_backward", "mor_expert_combine_backward_f32")


class MorMxOperand(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("ld_codes", C.c_int64), ("scales", C.c_void_p), ("ld_scales", C.c_int64),
                ("batch_codes", C.c_int64), ("batch_scales", C.c_int64)]


class MorMxParams(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("batch", C.c_int64), ("batch_x", C.c_int64),
                ("scale_rule", C.c_int32), ("rounding", C.c_int32), ("seed", C.c_uint64)]


class MorExpertOrder(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("top_k", C.c_int32), ("n_experts", C.c_int32), ("align", C.c_int32),
                ("capacity", C.c_int32), ("reserved", C.c_int32), ("offsets", C.c_void_p), ("slot_of", C.c_void_p),
                ("src", C.c_void_p)]


_lib = None


def load():
    """libmor.so with the signatures of this module's calls."""
    global _lib
    if _lib is None:
        L = binding.load()
        ptr, i64 = C.c_void_p, C.c_int64
        op = order = ptr                # addresses of a MorMxOperand, a MorExpertOrder
        signatures = {
            "mor_mx_quantize": ([ptr, ptr, op, op, order, ptr, ptr], C.c_int),
            "mor_mx_dequantize": ([i64, i64, i64, op, ptr, i64, i64, ptr], C.c_int),
            "mor_mx_product_workspace_bytes": ([i64, i64, i64], C.c_size_t),
            "mor_mx_product": ([i64, i64, i64, op, op, ptr, i64, C.c_int32, ptr, C.c_size_t, ptr], C.c_int),
            "mor_mx_product_rows": ([i64, i64, op, op, order, ptr, i64, C.c_int32, ptr], C.c_int),
            "mor_mx_product_depth": ([i64, i64, op, op, order, ptr, i64, i64, C.c_int32, ptr], C.c_int),
            "mor_expert_capacity": ([i64, i64, i64, i64], C.c_int64),
            "mor_expert_workspace_bytes": ([i64, i64, i64], C.c_size_t),
            "mor_expert_sort": ([ptr, order, ptr, C.c_size_t, ptr], C.c_int),
            "mor_expert_gather": ([ptr, i64, i64, order, ptr, i64, ptr], C.c_int),
            "mor_expert_combine": ([ptr, i64, i64, order, ptr, ptr, i64, ptr], C.c_int),
            "mor_expert_combine_f32": ([ptr, i64, i64, order, ptr, ptr, i64, C.c_int32, ptr], C.c_int),
            "mor_expert_combine_backward_f32": ([ptr, i64, ptr, i64, i64, order, ptr, ptr, i64, ptr, ptr], C.c_int),
            "mor_expert_combine_backward": ([ptr, i64, ptr, i64, i64, order, ptr, ptr, i64, ptr, ptr], C.c_int),
        }
        for name, (args, result) in signatures.items():
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, result
        _lib = L
    return _lib


def _device(where: str, *things) -> int:
    """Index of the device that all of ``things`` (tensors, operands, orders; None: not there) live on."""
    found = {t.get_device() for t in things if t is not None}
    if min(found) < 0:
        raise ValueError(f"{where}: all tensors must live in device memory")
    if len(found) > 1:
        raise ValueError(f"{where}: tensors on devices {sorted(found)}")
    return found.pop()


def _run(where: str, device: int, *args) -> None:
    """Calls the library with ``device`` as the current one and its current stream."""
    call = getattr(_lib or load(), where)
    if device == torch.cuda.current_device():
        rc = call(*args, binding._raw_stream(device) if binding._raw_stream is not None else binding._stream())
    else:
        with torch.cuda.device(device):
            rc = call(*args, binding._stream())
    if rc != 0:
        raise binding.MorError(rc, where)


def _matrix(t: torch.Tensor, name: str, types=(torch.bfloat16, torch.int16)) -> int:
    """Checks a matrix (or a batch of them) and returns the elements between its rows."""
    if t.dtype not in types:
        raise ValueError(f"{name}: {t.dtype} is not one of {types}")
    shape, stride = t.shape, t.stride()
    if len(shape) not in (2, 3) or (stride[-1] != 1 and shape[-1] > 1):
        raise ValueError(f"{name} must be two- or three-dimensional with unit stride along its rows")
    # the stride of a dimension of size one can be anything; that row's own length serves
    return stride[-2] if shape[-2] > 1 else shape[-1]


def _batch(t: torch.Tensor) -> tuple[int, int]:
    return (t.shape[0], t.stride(0) if t.shape[0] > 1 else 0) if t.dim() == 3 else (1, 0)


def _vector(t: torch.Tensor | None, name: str, dtype, n: int) -> None:
    if t is None:
        return
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be {n} contiguous elements of {dtype}")


@dataclass(frozen=True)
class MxOperand:
    """A 4-bit operand of ``rows`` x ``cols`` elements, or a batch of them (three-dimensional tensors)."""
    codes: torch.Tensor     # ([batch,] rows, 16 * blocks or more) uint8, two codes per byte
    scales: torch.Tensor    # ([batch,] rows, blocks or more) uint8, biased exponents
    rows: int
    cols: int

    def __post_init__(self):
        for t, name, least in ((self.codes, "codes", 16 * self.blocks), (self.scales, "scales", self.blocks)):
            if t.dtype != torch.uint8 or t.dim() not in (2, 3) or t.shape[-2] != self.rows or t.shape[-1] < least or t.stride(-1) != 1:
                raise ValueError(f"{name} must be uint8, ([batch,] {self.rows}, at least {least}), with unit stride along its rows")
        if self.codes.shape[:-1] != self.scales.shape[:-1]:
            raise ValueError("codes and scales must have the same batch and rows")
        if self.codes.device != self.scales.device:
            raise ValueError("codes and scales must live on one device")
        # a lone row's distance to the next can be anything; the bytes that its blocks take serve
        lone = self.rows == 1
        object.__setattr__(self, "batch", self.codes.shape[0] if self.codes.dim() == 3 else 1)
        object.__setattr__(self, "_index", self.codes.get_device())         # (its buffers do not change)
        object.__setattr__(self, "_struct", MorMxOperand(
            None, 16 * self.blocks if lone else self.codes.stride(-2), None, -(-self.blocks // 4) * 4 if lone else self.scales.stride(-2),
            self.codes.stride(0) if self.codes.dim() == 3 else 0, self.scales.stride(0) if self.scales.dim() == 3 else 0))

    @property
    def blocks(self) -> int:
        return -(-self.cols // BLOCK)

    def get_device(self) -> int:
        return self._index

    def struct(self) -> int:
        """Address of the operand's structure, valid as long as the operand."""
        struct = self._struct
        struct.codes, struct.scales = self.codes.data_ptr(), self.scales.data_ptr()
        return C.addressof(struct)


def alloc_operand(rows: int, cols: int, device, batch: int | None = None) -> MxOperand:
    blocks = -(-cols // BLOCK)
    lead = (rows,) if batch is None else (batch, rows)
    return MxOperand(torch.empty((*lead, 16 * blocks), dtype=torch.uint8, device=device),
                     torch.empty((*lead, -(-blocks // 4) * 4), dtype=torch.uint8, device=device), rows, cols)


@dataclass(frozen=True)
class ExpertOrder:
    """Tokens sorted by expert: buffers that :func:`mor_expert_sort` fills and the other calls read."""
    tokens: int
    top_k: int
    n_experts: int
    align: int
    capacity: int
    offsets: torch.Tensor   # (n_experts + 1,) int32, first slot of each expert
    slot_of: torch.Tensor   # (tokens * top_k,) int32, slot of each choice, -1: dropped
    src: torch.Tensor       # (capacity,) int32, choice in each slot, -1: empty
    workspace: torch.Tensor | None

    def __post_init__(self):
        _vector(self.offsets, "offsets", torch.int32, self.n_experts + 1)
        _vector(self.slot_of, "slot_of", torch.int32, self.tokens * self.top_k)
        _vector(self.src, "src", torch.int32, self.capacity)
        object.__setattr__(self, "_index", _device("ExpertOrder", self.offsets, self.slot_of, self.src, self.workspace))
        object.__setattr__(self, "_struct", MorExpertOrder(self.tokens, self.top_k, self.n_experts, self.align, self.capacity, 0))

    def get_device(self) -> int:
        return self._index

    def struct(self) -> int:
        """Address of the order's structure, valid as long as the order."""
        struct = self._struct
        struct.offsets, struct.slot_of, struct.src = self.offsets.data_ptr(), self.slot_of.data_ptr(), self.src.data_ptr()
        return C.addressof(struct)


def expert_capacity(tokens: int, top_k: int, n_experts: int, align: int = 128) -> int:
    return int(load().mor_expert_capacity(tokens, top_k, n_experts, align))


def alloc_order(tokens: int, top_k: int, n_experts: int, device, align: int = 128) -> ExpertOrder:
    """``align``: slots that an expert's segment is a multiple of; 128 for :func:`mor_mx_product_depth`, 1 where no gradient
    is wanted."""
    capacity = expert_capacity(tokens, top_k, n_experts, align)
    if capacity < 0:
        raise binding.MorError(2, "alloc_order")
    ints = lambda n: torch.empty(n, dtype=torch.int32, device=device)
    nbytes = int(load().mor_expert_workspace_bytes(tokens, top_k, n_experts))
    workspace = torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None
    return ExpertOrder(tokens, top_k, n_experts, align, capacity, ints(n_experts + 1), ints(tokens * top_k), ints(capacity), workspace)


def mor_mx_quantize(x: torch.Tensor, out: MxOperand | None = None, out_t: MxOperand | None = None, scale_rule: str = "floor",
                    rounding: str = "nearest", seed: int = 0, order: ExpertOrder | None = None, weights: torch.Tensor | None = None) -> None:
    """Quantise ``x`` ([batch,] rows, cols; BF16, or int16 holding its bits) into ``out`` and / or, transposed, ``out_t``.  With ``order`` the
    rows of the operands are its slots, each times its choice's weight if ``weights`` is given."""
    ld = _matrix(x, "x")
    rows, cols = x.shape[-2:]
    batch, batch_x = _batch(x)
    if order is not None:
        _vector(weights, "weights", torch.float32, order.tokens * order.top_k)
        slots = order.capacity
    else:
        slots = rows
    for operand, shape, name in ((out, (slots, cols), "out"), (out_t, (cols, slots), "out_t")):
        if operand is not None and ((operand.rows, operand.cols) != shape or operand.batch != batch):
            raise ValueError(f"{name} must be {batch} operand(s) of {shape[0]} x {shape[1]}")
    params = MorMxParams(rows, cols, ld, batch, batch_x, SCALE_RULE[scale_rule], ROUNDING[rounding], seed & 0xFFFFFFFFFFFFFFFF)
    device = x.get_device()
    if device < 0 or (out is not None and out._index != device) or (out_t is not None and out_t._index != device) or \
            (order is not None and order._index != device) or (weights is not None and weights.get_device() != device):
        _device("mor_mx_quantize", x, out, out_t, order, weights)
    _run("mor_mx_quantize", device, C.addressof(params), x.data_ptr(),
         out.struct() if out is not None else None, out_t.struct() if out_t is not None else None,
         order.struct() if order is not None else None, binding._ptr(weights))


def mor_mx_dequantize(operand: MxOperand, y: torch.Tensor) -> None:
    """``y`` ([batch,] rows, cols; BF16): what the operand stands for."""
    ld = _matrix(y, "y")
    batch, batch_y = _batch(y)
    if y.shape[-2:] != (operand.rows, operand.cols) or batch != operand.batch:
        raise ValueError(f"y must be {operand.batch} matrices of {operand.rows} x {operand.cols}")
    device = operand._index
    if device < 0 or y.get_device() != device:
        _device("mor_mx_dequantize", operand, y)
    _run("mor_mx_dequantize", device, operand.rows, operand.cols, batch, operand.struct(),
         y.data_ptr(), ld, batch_y)


_OUT = {torch.bfloat16: 0, torch.float32: 1}


def mor_mx_product_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(load().mor_mx_product_workspace_bytes(m, n, k))


def alloc_product_workspace(a: MxOperand, b: MxOperand, device) -> torch.Tensor | None:
    """Scratch of ``mor_mx_product(a, b, ...)``, None where it needs none."""
    nbytes = mor_mx_product_workspace_bytes(a.rows, b.rows, a.cols)
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def mor_mx_product(a: MxOperand, b: MxOperand, c: torch.Tensor, workspace: torch.Tensor | None = None) -> None:
    """``c`` (a.rows, b.rows; BF16 or float32) = a b^T."""
    ld = _matrix(c, "c", _OUT)
    if a.cols != b.cols or a.batch != 1 or b.batch != 1 or c.shape != (a.rows, b.rows):
        raise ValueError(f"shapes do not match: {a.rows} x {a.cols}, {b.rows} x {b.cols}, result {tuple(c.shape)}")
    device = a._index
    if device < 0 or b._index != device or c.get_device() != device or (workspace is not None and workspace.get_device() != device):
        _device("mor_mx_product", a, b, c, workspace)
    _run("mor_mx_product", device, a.rows, b.rows, a.cols, a.struct(), b.struct(), c.data_ptr(), ld,
         _OUT[c.dtype], binding._ptr(workspace), workspace.numel() if workspace is not None else 0)


def mor_mx_product_rows(a: MxOperand, b: MxOperand, order: ExpertOrder, c: torch.Tensor) -> None:
    """``c`` (capacity, b.rows): the slots' rows of ``a`` times their expert's operand of the batch ``b``, transposed."""
    ld = _matrix(c, "c", _OUT)
    if a.cols != b.cols or a.batch != 1 or a.rows != order.capacity or b.batch != order.n_experts or c.shape != (a.rows, b.rows):
        raise ValueError(f"shapes do not match: {a.rows} x {a.cols}, {b.batch} of {b.rows} x {b.cols}, {order.n_experts} experts, "
                         f"{order.capacity} slots, result {tuple(c.shape)}")
    device = a._index
    if device < 0 or b._index != device or order._index != device or c.get_device() != device:
        _device("mor_mx_product_rows", a, b, order, c)
    _run("mor_mx_product_rows", device, b.rows, a.cols, a.struct(), b.struct(), order.struct(),
         c.data_ptr(), ld, _OUT[c.dtype])


def mor_mx_product_depth(a: MxOperand, b: MxOperand, order: ExpertOrder, c: torch.Tensor) -> None:
    """``c`` (n_experts, a.rows, b.rows): for each expert a b^T summed over its slots, which are the columns of both."""
    ld = _matrix(c, "c", _OUT)
    if a.cols != order.capacity or b.cols != order.capacity or a.batch != 1 or b.batch != 1 or \
            c.dim() != 3 or c.shape != (order.n_experts, a.rows, b.rows):
        raise ValueError(f"shapes do not match: {a.rows} x {a.cols}, {b.rows} x {b.cols}, {order.n_experts} experts, "
                         f"{order.capacity} slots, result {tuple(c.shape)}")
    device = a._index
    if device < 0 or b._index != device or order._index != device or c.get_device() != device:
        _device("mor_mx_product_depth", a, b, order, c)
    _run("mor_mx_product_depth", device, a.rows, b.rows, a.struct(), b.struct(), order.struct(),
         c.data_ptr(), ld, _batch(c)[1], _OUT[c.dtype])


def mor_expert_sort(ids: torch.Tensor, order: ExpertOrder) -> None:
    """``ids`` (tokens, top_k) int32: the expert of each choice; outside [0, n_experts): dropped."""
    _vector(ids, "ids", torch.int32, order.tokens * order.top_k)
    ws = order.workspace
    device = order._index
    if ids.get_device() != device:
        _device("mor_expert_sort", ids, order)
    _run("mor_expert_sort", device, ids.data_ptr(), order.struct(), binding._ptr(ws),
         ws.numel() if ws is not None else 0)


def _rows(t: torch.Tensor | None, name: str, rows: int, d: int, types=(torch.bfloat16, torch.int16)) -> int:
    if t is None:
        return 0
    ld = _matrix(t, name, types)
    if t.shape != (rows, d):
        raise ValueError(f"{name} must be {rows} x {d}, not {tuple(t.shape)}")
    return ld


def mor_expert_gather(x: torch.Tensor, order: ExpertOrder, xs: torch.Tensor) -> None:
    """``xs`` (capacity, d): the token's row for every slot, zeros for empty ones."""
    d = x.shape[-1]
    ld_x, ld_xs = _rows(x, "x", order.tokens, d), _rows(xs, "xs", order.capacity, d)
    device = order._index
    if x.get_device() != device or xs.get_device() != device:
        _device("mor_expert_gather", x, order, xs)
    _run("mor_expert_gather", device, x.data_ptr(), ld_x, d, order.struct(), xs.data_ptr(), ld_xs)


_ROWS = (torch.bfloat16, torch.int16, torch.float32)


def mor_expert_combine(ys: torch.Tensor, order: ExpertOrder, weights: torch.Tensor | None, y: torch.Tensor) -> None:
    """``y`` (tokens, d): weighted sum of each token's rows of ``ys`` (capacity, d).  BF16, or rows in float32 and ``y`` in either."""
    d = ys.shape[-1]
    f32 = ys.dtype == torch.float32
    ld_ys, ld_y = _rows(ys, "ys", order.capacity, d, _ROWS), _rows(y, "y", order.tokens, d, _ROWS if f32 else _ROWS[:2])
    _vector(weights, "weights", torch.float32, order.tokens * order.top_k)
    where = "mor_expert_combine_f32" if f32 else "mor_expert_combine"
    device = order._index
    if ys.get_device() != device or y.get_device() != device or (weights is not None and weights.get_device() != device):
        _device(where, ys, order, weights, y)
    _run(where, device, ys.data_ptr(), ld_ys, d, order.struct(), binding._ptr(weights), y.data_ptr(), ld_y,
         *((int(y.dtype == torch.float32),) if f32 else ()))


def mor_expert_combine_backward(dy: torch.Tensor, ys: torch.Tensor | None, order: ExpertOrder, weights: torch.Tensor | None,
                                dys: torch.Tensor | None, dweights: torch.Tensor | None) -> None:
    """Gradients of :func:`mor_expert_combine`: ``dys`` (capacity, d; BF16) and ``dweights`` (tokens, top_k), either may be None."""
    d = dy.shape[-1]
    ld_dy, ld_ys, ld_dys = _rows(dy, "dy", order.tokens, d), _rows(ys, "ys", order.capacity, d, _ROWS), _rows(dys, "dys", order.capacity, d)
    _vector(weights, "weights", torch.float32, order.tokens * order.top_k)
    _vector(dweights, "dweights", torch.float32, order.tokens * order.top_k)
    where = "mor_expert_combine_backward_f32" if ys is not None and ys.dtype == torch.float32 else "mor_expert_combine_backward"
    device = _device(where, dy, ys, order, weights, dys, dweights)
    _run(where, device, dy.data_ptr(), ld_dy, binding._ptr(ys), ld_ys, d, order.struct(),
         binding._ptr(weights), binding._ptr(dys), ld_dys, binding._ptr(dweights))
