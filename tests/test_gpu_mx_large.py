"""The variants that large sizes take: reads and writes past the caches, several rows per lane, tiles of 128 sorted rows, several rounds per
workgroup of the sort, rows of experts' operands far apart.

Rounding to nearest depends on a row (transposed: on 32 rows) alone, so a large call has to give what calls of slices give that are
small enough for the other variants, which the tests of small sizes compare with the 64-bit model.  Stochastic and weighted
operands are compared with the model itself in sampled rows and columns.  Sums and scalar products: bounds as in the tests of small
sizes, (top_k + 1) 2^-24 or d 2^-24 of sum |terms| and one rounding to the result's type, evaluated in binary64 on the GPU."""
import numpy as np
import pytest
import torch

import mx_refmodel as R
from paper_2512_22804_amd import mx
from test_gpu_mx import close, random_operand
from test_gpu_mx_experts import make_order

pytestmark = pytest.mark.gpu
DEV = "cuda"
SLICE = 1024


def tensor(rows, cols, seed, pad=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    a = torch.randn(rows, cols + pad, generator=gen, device=DEV) * torch.exp(3 * torch.randn(rows, 1, generator=gen, device=DEV))
    a[torch.rand(rows, cols + pad, generator=gen, device=DEV) < 0.05] = 0.0
    return a.to(torch.bfloat16)[:, :cols]


def filled(rows, cols):
    op = mx.alloc_operand(rows, cols, DEV)
    op.codes.fill_(0xA5)
    op.scales.fill_(0xA5)
    return op


def same_rows(op, at, part):
    """Rows at .. of an operand are those of a smaller one."""
    n = part.rows
    assert torch.equal(op.codes[at:at + n], part.codes) and torch.equal(op.scales[at:at + n, :op.blocks], part.scales[:, :op.blocks])


def same_columns(op, at, part):
    """Columns at .. of an operand (at a multiple of 32) are those of a smaller one."""
    assert torch.equal(op.codes[:, at // 2:at // 2 + part.codes.shape[1]], part.codes)
    assert torch.equal(op.scales[:, at // 32:at // 32 + part.blocks], part.scales[:, :part.blocks])


def compare_slices(x, out, out_t):
    for at in range(0, x.shape[0], SLICE):
        part = x[at:at + SLICE]
        a, b = filled(part.shape[0], x.shape[1]), filled(x.shape[1], part.shape[0])
        mx.mor_mx_quantize(part, a, b)
        if out is not None:
            same_rows(out, at, a)
        if out_t is not None:
            same_columns(out_t, at, b)


def compare_samples(values, out, out_t, seed, rng, rule="floor"):
    """`values`: binary64 on the host; `seed`: of stochastic rounding, or None."""
    for op, v, form in ((out, values, 0), (out_t, values.T, 1)):
        if op is None:
            continue
        picked = np.unique(np.concatenate((rng.integers(0, op.rows, 30), [0, op.rows - 1])))
        random = R.random16(*v.shape, form, seed)[picked] if seed is not None else None
        codes, scales, _ = R.quantize(np.ascontiguousarray(v[picked]), rule, random)
        got = R.unpack_codes(op.codes[torch.from_numpy(picked).to(DEV)].cpu().numpy(), op.blocks * 32)
        assert np.array_equal(got[:, :op.cols], codes) and (got[:, op.cols:] == 0).all()
        assert np.array_equal(op.scales[torch.from_numpy(picked).to(DEV)].cpu().numpy()[:, :op.blocks], scales)


# past the caches from 16 MiB on where rows are whole lines (both forms and the transposed one alone); the same size in other rows
@pytest.mark.parametrize("form", ["both", "cols"])
@pytest.mark.parametrize("rows, cols, pad", [(8192, 4096, 0), (4100, 2048, 64), (4099, 2050, 0)])
def test_quantize_transposed(rows, cols, pad, form):
    x = tensor(rows, cols, 1, pad)
    out, out_t = filled(rows, cols) if form == "both" else None, filled(cols, rows)
    mx.mor_mx_quantize(x, out, out_t)
    compare_slices(x, out, out_t)


@pytest.mark.parametrize("form", ["both", "cols", "rows"])
@pytest.mark.parametrize("rows, cols", [(4224, 2048), (4227, 2050)])
def test_quantize_stochastic(rows, cols, form):
    x = tensor(rows, cols, 2)
    out, out_t = filled(rows, cols) if form != "cols" else None, filled(cols, rows) if form != "rows" else None
    mx.mor_mx_quantize(x, out, out_t, rounding="stochastic", seed=41)
    compare_samples(x.double().cpu().numpy(), out, out_t, 41, np.random.default_rng(0))


@pytest.mark.parametrize("rows, cols, pad", [(4099, 1100, 0), (4096, 4096, 8)])
def test_quantize_rows_of_many_elements(rows, cols, pad):
    x = tensor(rows, cols, 3, pad)
    out = filled(rows, cols)
    mx.mor_mx_quantize(x, out)
    compare_slices(x, out, None)


# above 4 M elements through the caches, and from 64 MiB on past them where rows are whole lines
@pytest.mark.parametrize("rows, cols, pad", [(4099, 1100, 3), (8192, 4096, 0), (8200, 4160, 0), (8192, 4096, 8)])
def test_dequantize(rows, cols, pad):
    x = tensor(rows, cols, 4)
    op = filled(rows, cols)
    mx.mor_mx_quantize(x, op)
    y = torch.full((rows + 1, cols + pad), 7.0, dtype=torch.bfloat16, device=DEV)
    mx.mor_mx_dequantize(op, y[:rows, :cols])
    assert (y[rows:] == 7.0).all() and (y[:, cols:] == 7.0).all()
    for at in range(0, rows, SLICE):
        part = mx.MxOperand(op.codes[at:at + SLICE], op.scales[at:at + SLICE], min(SLICE, rows - at), cols)
        back = torch.empty(part.rows, cols, dtype=torch.bfloat16, device=DEV)
        mx.mor_mx_dequantize(part, back)
        assert torch.equal(back, y[at:at + part.rows, :cols])
    picked = np.array([0, 1, rows // 2, rows - 1])
    assert np.array_equal(y[picked, :cols].double().cpu().numpy(), R.quantize(x[picked].double().cpu().numpy())[2])


def routed(tokens, top_k, experts, align, seed):
    rng = np.random.default_rng(seed)
    ids = rng.integers(0, experts, (tokens, top_k)).astype(np.int32)
    ids[rng.random(ids.shape) < 0.05] = -1
    return make_order(ids, experts, align)


def gathered(x, order):
    src = order.src.long()
    return torch.where((src >= 0)[:, None], x[src.clamp(min=0) // order.top_k], torch.zeros((), dtype=x.dtype, device=DEV))


# tokens quantised once for three slots each, several rows per lane; tiles of 128 slots
@pytest.mark.parametrize("form", ["rows", "cols", "both"])
def test_quantize_sorted(form):
    order = routed(1400, 3, 6, 128, 5)
    x = tensor(1400, 1100, 6)
    out, out_t = filled(order.capacity, 1100) if form != "cols" else None, filled(1100, order.capacity) if form != "rows" else None
    mx.mor_mx_quantize(x, out, out_t, order=order)
    compare_slices(gathered(x, order), out, out_t)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
def test_quantize_sorted_and_weighted(rounding, weighted):
    order = routed(4000, 2, 5, 128, 7)
    x = tensor(4000, 2100, 8)
    weights = torch.randn(4000, 2, generator=torch.Generator(device=DEV).manual_seed(9), device=DEV)
    assert order.capacity // 128 * -(-2100 // 128) > 1024                   # tiles of 128 slots in either rounding
    out, out_t = filled(order.capacity, 2100), filled(2100, order.capacity)
    mx.mor_mx_quantize(x, out, out_t, order=order, weights=weights if weighted else None, rounding=rounding, seed=43, scale_rule="ceil")
    rows = gathered(x, order).float()
    if weighted:
        rows = rows * torch.where(order.src >= 0, weights.reshape(-1)[order.src.long().clamp(min=0)], torch.ones((), device=DEV))[:, None]
    compare_samples(rows.double().cpu().numpy(), out, out_t, 43 if rounding == "stochastic" else None, np.random.default_rng(1), "ceil")


# 64 MiB of sorted rows in whole lines; the same in other rows
@pytest.mark.parametrize("d, pad", [(4096, 0), (4032, 64), (4090, 3)])
def test_gather_combine_and_gradients(d, pad):
    tokens, top_k = 4200, 2
    order = routed(tokens, top_k, 16, 128, 10)
    cap = order.capacity
    assert cap * d * 2 >= 1 << 26
    slots = order.slot_of.long().view(tokens, top_k)
    x, dy = tensor(tokens, d, 11, pad), tensor(tokens, d, 12, pad)
    weights = torch.randn(tokens, top_k, generator=torch.Generator(device=DEV).manual_seed(13), device=DEV)
    rows = lambda n, dtype=torch.bfloat16: torch.full((n + 1, d + pad), 7.0, dtype=dtype, device=DEV)

    def untouched(t, n):
        assert (t[n:] == 7.0).all() and (t[:, d:] == 7.0).all()

    xs = rows(cap)
    mx.mor_expert_gather(x, order, xs[:cap, :d])
    assert torch.equal(xs[:cap, :d], gathered(x, order))
    untouched(xs, cap)
    for rows_type in (torch.bfloat16, torch.float32):
        ys = tensor(cap, d, 14, pad) if rows_type == torch.bfloat16 else torch.randn(cap, d + pad, device=DEV)[:, :d]
        for y_type in (torch.bfloat16, torch.float32) if rows_type == torch.float32 else (torch.bfloat16,):
            for w in (weights, None):
                y = rows(tokens, y_type)
                mx.mor_expert_combine(ys, order, w, y[:tokens, :d])
                exact, total = torch.zeros(tokens, d, dtype=torch.float64, device=DEV), torch.zeros(tokens, d, dtype=torch.float64, device=DEV)
                for j in range(top_k):
                    term = torch.where((slots[:, j] >= 0)[:, None], ys[slots[:, j].clamp(min=0)].double(), 0.0)
                    term = term * w[:, j:j + 1].double() if w is not None else term
                    exact += term
                    total += term.abs()
                unit = 2.0 ** -8 if y_type == torch.bfloat16 else 2.0 ** -24
                assert ((y[:tokens, :d].double() - exact).abs() <= (top_k + 1) * 2.0 ** -24 * total + unit * exact.abs()).all()
                untouched(y, tokens)
        for form in ("both", "dys", "dweights"):
            dys, dw = rows(cap), torch.full((tokens, top_k), 9.0, device=DEV)
            mx.mor_expert_combine_backward(dy, ys, order, weights, dys[:cap, :d] if form != "dweights" else None, dw if form != "dys" else None)
            if form != "dweights":
                w = torch.where(order.src >= 0, weights.reshape(-1)[order.src.long().clamp(min=0)], torch.zeros((), device=DEV))
                want = gathered(dy, order).double() * w[:, None].double()
                assert ((dys[:cap, :d].double() - want).abs() <= 2.0 ** -8 * want.abs()).all()
                untouched(dys, cap)
            if form != "dys":
                for j in range(top_k):
                    terms = torch.where((slots[:, j] >= 0)[:, None], ys[slots[:, j].clamp(min=0)].double(), 0.0) * dy.double()
                    dot, size = terms.sum(1), terms.abs().sum(1)
                    assert ((dw[:, j].double() - dot).abs() <= d * 2.0 ** -24 * size + 2.0 ** -23 * dot.abs()).all()
                assert (dw[slots < 0] == 0).all()


@pytest.mark.parametrize("tokens, top_k, experts, align", [(150000, 2, 64, 128), (300001, 1, 7, 1), (90000, 6, 300, 16)])
def test_sort_of_many_choices(tokens, top_k, experts, align):
    """More than 2^18 choices: a workgroup takes them in several rounds."""
    rng = np.random.default_rng(tokens)
    p = np.exp(rng.standard_normal(experts))
    ids = rng.choice(experts, size=(tokens, top_k), p=p / p.sum()).astype(np.int32)
    ids[rng.random(ids.shape) < 0.1] = -1
    order = make_order(ids, experts, align)
    flat = ids.reshape(-1)
    kept = np.nonzero(flat >= 0)[0]
    by_expert = kept[np.argsort(flat[kept], kind="stable")]
    counts = np.bincount(flat[kept], minlength=experts)
    starts = np.concatenate(([0], np.cumsum(-(-counts // align) * align)))
    slot, src = np.full(flat.size, -1, np.int32), np.full(order.capacity, -1, np.int32)
    within = np.arange(by_expert.size) - np.repeat(np.cumsum(counts) - counts, counts)
    slot[by_expert] = starts[flat[by_expert]] + within
    src[slot[by_expert]] = by_expert
    assert np.array_equal(order.offsets.cpu().numpy(), starts)
    assert np.array_equal(order.slot_of.cpu().numpy(), slot) and np.array_equal(order.src.cpu().numpy(), src)


FAR = (1 << 23) + 16                    # bytes between rows from which 256 of them are out of reach of 32-bit offsets


def far_apart(op):
    lead = op.codes.shape[:-1]
    codes = torch.empty(*lead, FAR, dtype=torch.uint8, device=DEV)[..., :op.codes.shape[-1]]
    codes.copy_(op.codes)
    return mx.MxOperand(codes, op.scales, op.rows, op.cols)


@pytest.mark.parametrize("which", ["a", "b"])
def test_product_rows_far_apart(which):
    order = routed(60, 2, 3, 1, 15)
    a, av = random_operand(order.capacity, 200, 16)
    b, bv = random_operand(45, 200, 17, batch=3)
    c = torch.full((order.capacity + 1, 48), 7.0, device=DEV)
    mx.mor_mx_product_rows(far_apart(a) if which == "a" else a, far_apart(b) if which == "b" else b, order, c[:-1, :45])
    starts, got = order.offsets.cpu().numpy(), c.double().cpu().numpy()
    assert (got[starts[-1]:] == 7.0).all() and (got[:, 45:] == 7.0).all()
    for e in range(3):
        s = slice(starts[e], starts[e + 1])
        close(got[s, :45], av[s], bv[e], True, 200)


@pytest.mark.parametrize("which", ["a", "b"])
def test_product_depth_far_apart(which):
    order = routed(300, 2, 3, 128, 18)
    a, av = random_operand(40, order.capacity, 19)
    b, bv = random_operand(70, order.capacity, 20)
    c = torch.full((3, 41, 72), 7.0, device=DEV)
    mx.mor_mx_product_depth(far_apart(a) if which == "a" else a, far_apart(b) if which == "b" else b, order, c[:, :40, :70])
    starts, got = order.offsets.cpu().numpy(), c.double().cpu().numpy()
    assert (got[:, 40:] == 7.0).all() and (got[:, :, 70:] == 7.0).all()
    for e in range(3):
        s = slice(starts[e], starts[e + 1])
        close(got[e, :40, :70], av[:, s], bv[:, s], True, max(1, starts[e + 1] - starts[e]))
