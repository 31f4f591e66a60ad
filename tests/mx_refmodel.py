"""Plain 64-bit model of the microscaled 4-bit operands, of their products and of tokens sorted by expert (numpy, CPU)."""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def random16(rows, cols, form, seed, batch=0):
    """16 random bits per element (Philox 4x32, seven rounds)."""
    groups = -(-cols // 8)
    c = [np.tile(np.arange(groups, dtype=np.uint64), rows), np.repeat(np.arange(rows, dtype=np.uint64), groups),
         np.full(rows * groups, batch, np.uint64), np.full(rows * groups, form, np.uint64)]
    k = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(7):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = [h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))]
    return np.stack(halves, 1).reshape(rows, groups * 8)[:, :cols].astype(np.int64)


def quantize(x, rule="floor", random=None):
    """(codes [rows, cols], bytes [rows, blocks], values [rows, cols]) of float64 rows that are exact in binary32."""
    rows, cols = x.shape
    blocks = -(-cols // BLOCK)
    wide = np.zeros((rows, blocks * BLOCK))
    wide[:, :cols] = x
    wide = wide.reshape(rows, blocks, BLOCK)
    bad = ~np.isfinite(wide).all(axis=2)
    amax = np.abs(np.where(bad[..., None], 1.0, wide)).max(axis=2)
    mantissa, exponent = np.frexp(amax)                        # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = exponent - 3 + ((mantissa > 0.75) if rule == "ceil" else 0)
    e = np.clip(np.where(amax == 0, 0, e), -127, 127)
    with np.errstate(invalid="ignore"):
        y = np.ldexp(np.abs(wide), -e[..., None])
        distance = np.abs(np.minimum(y, 6.0)[..., None] - GRID)
    if random is None:
        # the nearest; of two equally near the even code
        code = np.where(distance[..., 1::2].min(-1) < distance[..., 0::2].min(-1), 2 * distance[..., 1::2].argmin(-1) + 1,
                        2 * distance[..., 0::2].argmin(-1))
    else:
        r = np.zeros((rows, blocks * BLOCK), np.int64)
        r[:, :cols] = random
        r = r.reshape(wide.shape)
        below = np.clip(np.searchsorted(GRID, y, side="right") - 1, 0, 6)
        step = GRID[below + 1] - GRID[below]
        with np.errstate(invalid="ignore"):
            code = np.minimum(below + ((y - GRID[below]) / step + r / 65536.0 >= 1.0), 7)
    code = np.where(bad[..., None], 0, code)
    values = np.copysign(GRID[code], wide) * np.ldexp(1.0, e)[..., None]
    values[bad] = np.nan
    sign = np.where(np.signbit(wide) & ~bad[..., None], 8, 0)
    return ((code | sign).reshape(rows, -1)[:, :cols], np.where(bad, 255, e + 127).astype(np.uint8),
            values.reshape(rows, -1)[:, :cols])


def unpack_codes(codes, cols):
    """Nibbles [rows, cols] of packed rows."""
    return np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1)[:, :cols]


def stand_for(codes, scales, cols):
    """Values [rows, cols] of packed codes and bytes."""
    nibbles = unpack_codes(codes, cols).astype(np.int64)
    values = np.where(nibbles >= 8, -1.0, 1.0) * GRID[nibbles & 7]
    blocks = -(-cols // BLOCK)
    scale = np.ldexp(1.0, scales[:, :blocks].astype(np.int64) - 127)
    scale[scales[:, :blocks] == 255] = np.nan
    return values * np.repeat(scale, BLOCK, axis=1)[:, :cols]


def sort(ids, n_experts, align, capacity):
    """Segment starts, slot of each choice, choice in each slot."""
    flat = ids.reshape(-1)
    lists = [[i for i in range(flat.size) if flat[i] == e] for e in range(n_experts)]
    starts, slot, src = [0], np.full(flat.size, -1, np.int32), np.full(capacity, -1, np.int32)
    for members in lists:
        for j, i in enumerate(members):
            slot[i] = starts[-1] + j
            src[starts[-1] + j] = i
        starts.append(starts[-1] + -(-len(members) // align) * align)
    return np.array(starts, np.int32), slot, src
