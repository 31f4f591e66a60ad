"""Microscaled 4-bit operands on the GPU: quantisation and products against the 64-bit model (tests/mx_refmodel.py).

Codes, scales and de-quantised values have to be equal.  Products: the sums run in binary32, one instruction adding 128
products; with S = sum |a b| the result is within (K / 128 + 2) 2^-22 S of the exact one (each instruction rounds or aligns
its terms and the running sum within 2 units of 2^-23 of their magnitudes), plus half a unit of the result's type.
"""
import numpy as np
import pytest
import torch

import mx_refmodel as R
from paper_2512_22804_amd import binding as B
from paper_2512_22804_amd import mx
from paper_2512_22804_amd import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda"


def bf16(values):
    """BF16 tensor on the GPU and its values in binary64."""
    t = torch.from_numpy(np.ascontiguousarray(values, dtype=np.float32)).to(torch.bfloat16)
    return t.to(DEV), t.double().numpy()


def operand_values(rows, cols, seed):
    rng = np.random.default_rng(seed)
    a = rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)) * 3)
    a[rng.random((rows, cols)) < 0.05] = 0.0
    a[rng.random((rows, cols)) < 0.02] *= -0.0
    return a


def guarded(rows, cols, batch=None):
    """An operand whose buffers end (and whose rows are apart) in bytes that nobody may write."""
    blocks = -(-cols // 32)
    lead = (rows,) if batch is None else (batch, rows)
    codes = torch.full((*lead, 16 * blocks + 32), 0xA5, dtype=torch.uint8, device=DEV)
    scales = torch.full((*lead, (blocks + 3) // 4 * 4 + 8), 0xA5, dtype=torch.uint8, device=DEV)
    return mx.MxOperand(codes, scales, rows, cols)


def check_operand(op, want_codes, want_scales, batch=None):
    codes = (op.codes if batch is None else op.codes[batch]).cpu().numpy()
    scales = (op.scales if batch is None else op.scales[batch]).cpu().numpy()
    blocks = op.blocks
    assert np.array_equal(scales[:, :blocks], want_scales)
    got = R.unpack_codes(codes[:, :16 * blocks], 32 * blocks)
    assert np.array_equal(got[:, :op.cols], want_codes)
    assert (got[:, op.cols:] == 0).all()                       # what the last block lacks
    assert (codes[:, 16 * blocks:] == 0xA5).all() and (scales[:, (blocks + 3) // 4 * 4:] == 0xA5).all()


SIZES = [(1, 1), (1, 31), (2, 32), (1, 4097), (3, 129), (17, 200), (128, 128), (129, 257), (300, 96), (40, 1000), (257, 33)]


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("rule", ["floor", "ceil"])
@pytest.mark.parametrize("rows, cols", SIZES)
def test_quantize_both_forms(rows, cols, rule, rounding):
    print(f"[mx] quantize {rows}x{cols} {rule} {rounding}", flush=True)
    x, v = bf16(operand_values(rows, cols, rows * 1000 + cols))
    seed = 0x1234567890ABCDEF
    random = (lambda r, c, form: R.random16(r, c, form, seed)) if rounding == "stochastic" else (lambda *a: None)
    want = R.quantize(v, rule, random(rows, cols, 0))
    want_t = R.quantize(v.T, rule, random(cols, rows, 1))
    for form in ("both", "rows", "cols"):
        out = guarded(rows, cols) if form != "cols" else None
        out_t = guarded(cols, rows) if form != "rows" else None
        mx.mor_mx_quantize(x, out, out_t, scale_rule=rule, rounding=rounding, seed=seed)
        for op, (codes, scales, values) in ((out, want), (out_t, want_t)):
            if op is None:
                continue
            check_operand(op, codes, scales)
            y = torch.full((op.rows, op.cols + 3), 7.0, dtype=torch.bfloat16, device=DEV)
            mx.mor_mx_dequantize(op, y[:, :op.cols])
            got = y.double().cpu().numpy()
            assert np.array_equal(got[:, :op.cols], values, equal_nan=True) and (got[:, op.cols:] == 7.0).all()


@pytest.mark.parametrize("pad, shift", [(0, 0), (8, 0), (3, 0), (0, 1), (5, 3)])
def test_quantize_strides_and_alignment(pad, shift):
    rows, cols = 70, 133
    buf = torch.randn(rows * (cols + pad) + 16, device=DEV).to(torch.bfloat16)
    x = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    v = x.double().cpu().numpy()
    out, out_t = guarded(rows, cols), guarded(cols, rows)
    mx.mor_mx_quantize(x, out, out_t)
    check_operand(out, *R.quantize(v)[:2])
    check_operand(out_t, *R.quantize(v.T)[:2])
    ybuf = torch.zeros(rows * (cols + pad) + 16, dtype=torch.bfloat16, device=DEV)
    y = ybuf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    mx.mor_mx_dequantize(out, y)
    assert np.array_equal(y.double().cpu().numpy(), R.quantize(v)[2])
    assert int((ybuf != 0).sum()) == int((y != 0).sum())


@pytest.mark.parametrize("rule", ["floor", "ceil"])
@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
def test_quantize_every_pattern(rule, rounding):
    """All 65536 BF16 patterns, in blocks with a companion that sets the amax: 2^0 .. 2^3 above, or none."""
    bits = np.arange(65536, dtype=np.uint16)
    x = np.zeros((65536 // 8, 32), np.uint16)
    x[:, :8] = bits.reshape(-1, 8)
    f = W.bf16_bits_to_f32(x)
    with np.errstate(all="ignore"):
        top = np.abs(f).max(axis=1)
        companion = top * np.exp2(np.arange(len(top)) % 5 - 1).astype(np.float32)
    companion = np.where(np.isfinite(companion), companion, 0)
    x[:, 31] = W.f32_to_bf16_bits(np.where(np.arange(len(top)) % 5 == 0, 0, companion).astype(np.float32))
    t = torch.from_numpy(x.view(np.int16)).to(DEV)
    v = W.bf16_bits_to_f32(x).astype(np.float64)
    random = R.random16(*x.shape, 0, 99) if rounding == "stochastic" else None
    out = guarded(*x.shape)
    mx.mor_mx_quantize(t, out, scale_rule=rule, rounding=rounding, seed=99)
    codes, scales, values = R.quantize(v, rule, random)
    check_operand(out, codes, scales)
    values = np.where(np.abs(values) >= 2.0 ** 128, np.copysign(np.inf, values), values)   # the largest numbers round up to 2^128
    y = torch.empty(x.shape, dtype=torch.bfloat16, device=DEV)
    mx.mor_mx_dequantize(out, y)
    assert np.array_equal(y.double().cpu().numpy(), values, equal_nan=True)


def test_quantize_blocks_that_are_not_finite():
    x = torch.randn(4, 96, device=DEV).to(torch.bfloat16)
    x[1, 40], x[2, 0], x[3, 95] = float("inf"), float("nan"), float("-inf")
    out, out_t = guarded(4, 96), guarded(96, 4)
    mx.mor_mx_quantize(x, out, out_t)
    v = x.double().cpu().numpy()
    check_operand(out, *R.quantize(v)[:2])
    check_operand(out_t, *R.quantize(v.T)[:2])
    assert (out.scales[:, :3] == 255).sum().item() == 3


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
def test_quantize_batch(rounding):
    x, v = bf16(operand_values(3 * 50, 70, 5))
    x, v = x.view(3, 50, 70), v.reshape(3, 50, 70)
    out, out_t = guarded(50, 70, batch=3), guarded(70, 50, batch=3)
    mx.mor_mx_quantize(x, out, out_t, rounding=rounding, seed=3)
    y = torch.zeros(3, 50, 72, dtype=torch.bfloat16, device=DEV)[:, :, :70]
    mx.mor_mx_dequantize(out, y)
    for z in range(3):
        r, rt = ((R.random16(50, 70, 0, 3, z), R.random16(70, 50, 1, 3, z)) if rounding == "stochastic" else (None, None))
        want = R.quantize(v[z], "floor", r)
        check_operand(out, *want[:2], batch=z)
        check_operand(out_t, *R.quantize(v[z].T, "floor", rt)[:2], batch=z)
        assert np.array_equal(y[z].double().cpu().numpy(), want[2])


def test_quantize_rows_far_apart():
    """Byte offsets beyond 32 bits."""
    ld = (1 << 31) + 24
    buf = torch.empty(2 * ld, dtype=torch.bfloat16, device=DEV)
    x = buf.view(2, ld)[:, :200]
    x.copy_(torch.randn(2, 200, device=DEV))
    out, out_t = guarded(2, 200), guarded(200, 2)
    mx.mor_mx_quantize(x, out, out_t)
    v = x.double().cpu().numpy()
    check_operand(out, *R.quantize(v)[:2])
    check_operand(out_t, *R.quantize(v.T)[:2])


# ---- products ----------------------------------------------------------------------------------------------------------

def random_operand(rows, cols, seed, batch=None, spread=6):
    """A packed operand with arbitrary codes and scales of a range of 2 * spread binades, and its values."""
    rng = np.random.default_rng(seed)
    blocks = -(-cols // 32)
    lead = (rows,) if batch is None else (batch, rows)
    codes = rng.integers(0, 256, (*lead, 16 * blocks), dtype=np.uint8)
    if cols % 32:
        nibbles = np.stack((codes & 15, codes >> 4), -1).reshape(*lead, -1)
        nibbles[..., cols:] = 0
        codes = (nibbles[..., 0::2] | (nibbles[..., 1::2] << 4)).astype(np.uint8)
    scales = rng.integers(127 - spread, 127 + spread + 1, (*lead, (blocks + 3) // 4 * 4), dtype=np.uint8)
    op = mx.MxOperand(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV), rows, cols)
    flat = R.stand_for(codes.reshape(-1, 16 * blocks), scales.reshape(-1, scales.shape[-1]), cols)
    return op, flat.reshape(*lead, cols)


def close(got, a, b, f32, k):
    exact = a @ b.T
    total = np.abs(a) @ np.abs(b).T
    bound = (k / 128 + 2) * 2.0 ** -22 * total + np.abs(exact) * (2.0 ** -23 if f32 else 2.0 ** -8)
    off = np.abs(got - exact) > bound
    assert not off.any(), f"{off.sum()} of {off.size} off, first at {np.argwhere(off)[0]}: {got[off][0]} for {exact[off][0]}"


def product(a, b, dtype, **kw):
    c = torch.full((a.rows + 1, b.rows + 5), 7.0, dtype=dtype, device=DEV)
    ws = mx.alloc_product_workspace(a, b, DEV)
    if ws is not None:
        ws.fill_(0xFF)
    mx.mor_mx_product(a, b, c[:a.rows, :b.rows], ws)
    assert (c[a.rows:] == 7.0).all() and (c[:, b.rows:] == 7.0).all()
    return c[:a.rows, :b.rows].double().cpu().numpy()


PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 300, 4096), (2, 17, 33), (5, 1000, 1500), (16, 64, 128), (17, 128, 160), (33, 65, 127), (64, 512, 256),
            (100, 40, 5000), (128, 128, 128), (129, 257, 513), (200, 1, 640), (256, 256, 256), (257, 512, 1024), (300, 400, 4130),
            (512, 768, 2048), (1000, 130, 96), (2100, 2050, 300),
            # parts of the depth on different workgroups, the last one shorter, and a result joined from them
            (70, 100, 4096), (100, 257, 8200), (300, 130, 6000)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m, n, k", PRODUCTS)
def test_product(m, n, k, dtype):
    print(f"[mx] product {m}x{n}x{k} {dtype}", flush=True)
    a, av = random_operand(m, k, m + 7 * k)
    b, bv = random_operand(n, k, n + 11 * k)
    close(product(a, b, dtype), av, bv, dtype == torch.float32, k)


def test_product_is_repeatable():
    for m, n, k in ((1, 2000, 4096), (40, 512, 8192), (300, 300, 4096)):
        a, b = random_operand(m, k, 1)[0], random_operand(n, k, 2)[0]
        first = product(a, b, torch.float32)
        for _ in range(3):
            assert np.array_equal(first, product(a, b, torch.float32))


@pytest.mark.parametrize("m", [1, 40, 300])
def test_product_scales_at_the_ends(m):
    """Scales from 2^-127 to 2^127, whose product stays in range, and NaN bytes, whose rows of the result are NaN."""
    k, n = 160, 70
    a, _ = random_operand(m, k, 3)
    b, _ = random_operand(n, k, 4)
    a.scales.fill_(0)
    b.scales.fill_(254)
    values = lambda op: R.stand_for(op.codes.cpu().numpy(), op.scales.cpu().numpy(), k)
    close(product(a, b, torch.float32), values(a), values(b), True, k)
    a.scales.fill_(127)
    b.scales.fill_(127)
    a.scales[0, 1] = 255
    b.scales[n - 1, 4] = 255
    got, want = product(a, b, torch.float32), values(a) @ values(b).T
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(got[0]).all() and np.isnan(got[:, n - 1]).all()


@pytest.mark.parametrize("m", [1, 300])
def test_product_reads_no_padding(m):
    """What lies behind the blocks of a row (codes and scales) changes nothing, whatever it holds."""
    k, n = 4130, 200
    a, av = random_operand(m, k, 5)
    b, bv = random_operand(n, k, 6)
    wide = []
    for op in (a, b):
        codes = torch.full((op.rows, op.codes.shape[1] + 160), 0x77, dtype=torch.uint8, device=DEV)
        scales = torch.full((op.rows, op.scales.shape[1] + 20), 255, dtype=torch.uint8, device=DEV)
        codes[:, :op.codes.shape[1]] = op.codes
        scales[:, :op.blocks] = op.scales[:, :op.blocks]
        wide.append(mx.MxOperand(codes, scales, op.rows, k))
    close(product(*wide, torch.float32), av, bv, True, k)


def test_product_rows_far_apart():
    ld = (1 << 31) + 64
    codes = torch.empty(2 * ld, dtype=torch.uint8, device=DEV).view(2, ld)
    b, bv = random_operand(2, 500, 8)
    codes[:, :b.codes.shape[1]] = b.codes
    far = mx.MxOperand(codes, b.scales, 2, 500)
    a, av = random_operand(3, 500, 9)
    close(product(a, far, torch.float32), av, bv, True, 500)
    a, av = random_operand(300, 500, 9)
    close(product(a, far, torch.float32), av, bv, True, 500)


def test_product_of_quantised_operands_is_the_linear_layer():
    """Forward and both gradients of one linear layer from BF16 tensors."""
    t, h, w = 150, 200, 330
    x, xv = bf16(operand_values(t, h, 1))
    wt, wv = bf16(operand_values(w, h, 2))
    dy, gv = bf16(operand_values(t, w, 3))
    ops = {}
    for name, src in (("x", x), ("w", wt), ("g", dy)):
        ops[name], ops[name + "t"] = mx.alloc_operand(*src.shape, DEV), mx.alloc_operand(src.shape[1], src.shape[0], DEV)
        mx.mor_mx_quantize(src, ops[name], ops[name + "t"])
    q = lambda v: R.quantize(v)[2]
    close(product(ops["x"], ops["w"], torch.float32), q(xv), q(wv), True, h)
    close(product(ops["g"], ops["wt"], torch.float32), q(gv), q(wv.T), True, w)
    close(product(ops["gt"], ops["xt"], torch.float32), q(gv.T), q(xv.T), True, t)


def test_other_stream_and_graph():
    """The calls run on the current stream, and inside a captured graph, replayed on new inputs."""
    t, h, w = 64, 512, 256
    x = torch.randn(t, h, device=DEV).to(torch.bfloat16)
    weight = torch.randn(w, h, device=DEV).to(torch.bfloat16)
    xq, wq, y = mx.alloc_operand(t, h, DEV), mx.alloc_operand(w, h, DEV), torch.empty(t, w, device=DEV)
    ws = mx.alloc_product_workspace(xq, wq, DEV)
    mx.mor_mx_quantize(weight, wq)

    def step():
        mx.mor_mx_quantize(x, xq)
        mx.mor_mx_product(xq, wq, y, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    want = y.clone()
    y.zero_()
    step()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        x.copy_(torch.randn(t, h, device=DEV))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, y)


def test_refused_calls_leave_the_results():
    a, b = random_operand(8, 64, 1)[0], random_operand(8, 64, 2)[0]
    with pytest.raises(ValueError):
        mx.mor_mx_product(a, b, torch.empty(8, 9, device=DEV))
    with pytest.raises(ValueError):
        mx.mor_mx_product(a, random_operand(8, 96, 2)[0], torch.empty(8, 8, device=DEV))
    with pytest.raises(ValueError):
        mx.mor_mx_quantize(torch.zeros(8, 64, device=DEV), a)              # float32
    with pytest.raises(ValueError):
        mx.mor_mx_quantize(torch.zeros(64, 8, device=DEV, dtype=torch.bfloat16).t(), a)
    with pytest.raises(B.MorError) as e:
        mx.mor_mx_quantize(torch.zeros(8, 64, device=DEV, dtype=torch.bfloat16))
    assert e.value.status == 1
