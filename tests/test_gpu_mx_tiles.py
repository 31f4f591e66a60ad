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
