"""Products of more tiles than the GPU has compute units: workgroups that take several, quarters of tiles in the last round, experts of
very different sizes.  Bounds as for the products of other sizes."""
import numpy as np
import pytest
import torch

import mx_refmodel as R
from paper_2512_22804_amd import mx
from test_gpu_mx import close, product, random_operand
from test_gpu_mx_experts import make_order

pytestmark = pytest.mark.gpu
DEV = "cuda"


# 256 x 256 tiles: 17 x 16 (272: a round and quarters of 16), 16 x 20 (a round and 64), 18 x 18 + edges (whole tiles twice), 33 x 16
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m, n, k", [(4200, 4090, 512), (4096, 5120, 700), (4500, 4400, 300), (8200, 4096, 256), (4097, 4097, 33)])
def test_many_tiles(m, n, k, dtype):
    a, av = random_operand(m, k, 1, spread=3)
    b, bv = random_operand(n, k, 2, spread=3)
    close(product(a, b, dtype), av, bv, dtype == torch.float32, k)


SKEWS = {"even": lambda e: np.ones(e), "one": lambda e: np.eye(e)[e // 2] + 1e-9, "falling": lambda e: 0.7 ** np.arange(e)}


def skewed(tokens, top_k, experts, skew, seed):
    p = SKEWS[skew](experts)
    return np.random.default_rng(seed).choice(experts, size=(tokens, top_k), p=p / p.sum()).astype(np.int32)


@pytest.mark.parametrize("skew", SKEWS)
@pytest.mark.parametrize("tokens, top_k, experts, align, n, k", [(4000, 2, 16, 128, 2300, 260), (3000, 3, 8, 1, 2048, 512), (9000, 1, 70, 1, 1100, 96)])
def test_rows_of_experts_of_all_sizes(tokens, top_k, experts, align, n, k, skew):
    order = make_order(skewed(tokens, top_k, experts, skew, 3), experts, align)
    starts = order.offsets.cpu().numpy()
    a, av = random_operand(order.capacity, k, 4, spread=3)
    b, bv = random_operand(n, k, 5, batch=experts, spread=3)
    c = torch.full((order.capacity, n), 7.0, device=DEV)
    mx.mor_mx_product_rows(a, b, order, c)
    got = c.double().cpu().numpy()
    for e in range(experts):
        s = slice(starts[e], starts[e + 1])
        close(got[s], av[s], bv[e], True, k)
    assert (got[starts[-1]:] == 7.0).all()


@pytest.mark.parametrize("skew", SKEWS)
@pytest.mark.parametrize("tokens, top_k, experts, m, n", [(1500, 2, 5, 520, 1030), (700, 1, 37, 250, 600), (2000, 2, 3, 2100, 2050), (300, 2, 70, 130, 100)])
def test_depths_of_experts_of_all_sizes(tokens, top_k, experts, m, n, skew):
    order = make_order(skewed(tokens, top_k, experts, skew, 6), experts, 128)
    starts = order.offsets.cpu().numpy()
    a, av = random_operand(m, order.capacity, 7, spread=3)
    b, bv = random_operand(n, order.capacity, 8, spread=3)
    c = torch.full((experts, m, n), 7.0, device=DEV)
    mx.mor_mx_product_depth(a, b, order, c)
    got = c.double().cpu().numpy()
    for e in range(experts):
        s = slice(starts[e], starts[e + 1])
        close(got[e], av[:, s], bv[:, s], True, starts[e + 1] - starts[e])


# few rows against many, 16, 32 or 64 of them to a workgroup; more than 32 rows and a long depth
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m, n, k", [(3, 20500, 96), (4, 20481, 33), (5, 10300, 130), (16, 5200, 700), (20, 10250, 96), (32, 5203, 1030), (40, 10245, 200),
                                     (64, 6001, 513), (33, 100, 10400), (64, 3001, 10300), (64, 300, 10240)])
def test_few_rows(m, n, k, dtype):
    a, av = random_operand(m, k, 9, spread=3)
    b, bv = random_operand(n, k, 10, spread=3)
    close(product(a, b, dtype), av, bv, dtype == torch.float32, k)


@pytest.mark.parametrize("tokens, top_k, experts, n, k", [(5, 2, 6, 2100, 140), (1, 2, 30, 5201, 64), (60, 1, 5, 2045, 520), (30, 3, 8, 700, 1100), (63, 1, 5, 300, 96)])
def test_few_rows_of_experts(tokens, top_k, experts, n, k):
    order = make_order(skewed(tokens, top_k, experts, "falling", 11), experts, 1)
    starts = order.offsets.cpu().numpy()
    a, av = random_operand(order.capacity, k, 12, spread=3)
    b, bv = random_operand(n, k, 13, batch=experts, spread=3)
    c = torch.full((order.capacity + 1, n), 7.0, device=DEV)
    mx.mor_mx_product_rows(a, b, order, c[:-1])
    got = c.double().cpu().numpy()
    assert (got[-1] == 7.0).all()
    for e in range(experts):
        s = slice(starts[e], starts[e + 1])
        close(got[s], av[s], bv[e], True, k)


# transposed forms in tiles of 128 rows and of 32, weighted or not, in batches; the last tile of rows and of columns short
@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("batch, rows, cols", [(1, 4200, 1030), (1, 33, 33000), (3, 500, 700), (9, 500, 1003), (1, 8300, 2100), (1, 31, 5), (2, 1, 300)])
def test_transposed_forms(batch, rows, cols, rounding):
    rng = np.random.default_rng(rows)
    bits = rng.integers(0, 2 ** 16, (batch, rows, cols)).astype(np.uint16)
    bits[(bits & 0x7F80) == 0x7F80] = 0x3F80
    values = (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    values = np.where(np.abs(values) < 2.0 ** -100, 0.0, values)
    bits = np.where(values == 0.0, 0, bits).astype(np.uint16)
    x = torch.from_numpy(bits.view(np.int16)).to(DEV)
    out, out_t = mx.alloc_operand(rows, cols, DEV, batch=batch), mx.alloc_operand(cols, rows, DEV, batch=batch)
    for t in (out.codes, out.scales, out_t.codes, out_t.scales):
        t.fill_(0xA5)
    mx.mor_mx_quantize(x, out, out_t, rounding=rounding, seed=77)
    alone = mx.alloc_operand(cols, rows, DEV, batch=batch)
    mx.mor_mx_quantize(x, None, alone, rounding=rounding, seed=77)
    blocks = -(-rows // 32)
    assert torch.equal(alone.codes, out_t.codes) and torch.equal(alone.scales[..., :blocks], out_t.scales[..., :blocks])
    for z in range(0, batch, 4):
        for op, v, form in ((out, values[z], 0), (out_t, values[z].T, 1)):
            noise = R.random16(*v.shape, form, 77, z) if rounding == "stochastic" else None
            codes, scales, _ = R.quantize(v, "floor", noise)
            got = R.unpack_codes(op.codes[z].cpu().numpy(), op.codes.shape[-1] * 2)
            assert np.array_equal(got[:, :v.shape[1]], codes) and (got[:, v.shape[1]:] == 0).all()
            assert np.array_equal(op.scales[z].cpu().numpy()[:, :scales.shape[1]], scales)


# 256 x 256 tiles whose last round is cut in halves: 24 x 16 (384), 16 x 23 with edges (a round and 112), 45 x 8 with an edge (104)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("m, n, k", [(6144, 4096, 300), (4090, 5802, 520), (11400, 2047, 96)])
def test_tiles_in_halves(m, n, k, dtype):
    a, av = random_operand(m, k, 14, spread=3)
    b, bv = random_operand(n, k, 15, spread=3)
    close(product(a, b, dtype), av, bv, dtype == torch.float32, k)
