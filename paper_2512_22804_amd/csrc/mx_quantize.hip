// Quantisation of BF16 operands to microscaled 4 bits (rows, transposed, or both from one read) and back.
#include "mx_device.h"
#include "mx_launch.h"

namespace mor {
namespace {

constexpr int64_t kManyElements = 1 << 22;  // from here on a lane takes several rows
constexpr int kTileCols = 128;          // columns of a workgroup's tile: 16 lanes of 8 elements

// One workgroup: RPT * 16 rows x 128 columns, 256 lanes.  Lane t holds 8 columns (16 bytes) of RPT rows; a block of the row
// form is then 4 neighbouring lanes.  For the transposed form (T) the tile goes through LDS, and lane t takes a pair of columns over
// 4 RPT rows.  RPT = 8: a block's 32 rows, so that its amax needs no other lane and its 16 bytes are one store; four neighbouring
// lanes fill 64 bytes of an output row.  RPT = 2, for tensors of few tiles: 8 rows, four neighbouring lanes share a block, and a
// lane's chain of work is a quarter as long.  The rows are rotated by 16 dwords every 4 RPT of them: those that
// neighbouring lanes read then lie in different banks.
//
// Rounding to nearest is bound by memory (14336 x 4096: rows 31 us, transposed 32, both from one read 41 us = 4.3 TB/s), stochastic rounding
// by the vector unit (40, 40 and 63 us): a generator's seven rounds for eight elements and a dozen instructions for each.  Both forms
// in one launch read the tensor once, and a lane's eight rows are in flight together; tiles half as wide, twice as many on a
// CU, were slower (48 us for both).  Weighted rows are scaled in binary32 and not rounded in between (18432 x 2048 gathered, both
// forms, stochastic: 60 us: a slot, its choice's weight and its token's row are loads that wait for each other).
template <int RPT, bool ROWS, bool T, bool SR, bool WEIGHTED, bool STREAM>
__global__ __launch_bounds__(256, T && WEIGHTED ? 3 : 1) void k_mx_quantize(MxQuantArgs a, uint32_t col_tiles) {
    static_assert(!T || RPT == 8 || RPT == 2, "the transposed form works on tiles of 128 or 32 rows");
    constexpr int kRows = T ? 4 * RPT : 8;              // of a lane in the transposed form
    __shared__ __align__(16) uint32_t tile[T ? RPT * 16 * 64 : 4];
    __shared__ __align__(16) float row_weight[WEIGHTED ? RPT * 16 : 1];
    const int t = threadIdx.x;
    const uint32_t tile_id = tile_of(blockIdx.x, gridDim.x), ct = tile_id % col_tiles;
    const int64_t rt = tile_id / col_tiles;
    const int64_t c0 = (int64_t)ct * kTileCols, r0 = rt * (RPT * 16);
    const uint32_t z = blockIdx.z;
    const uint16_t* x = a.x + (int64_t)z * a.batch_x;
    const int64_t c = c0 + (t & 15) * 8;
    const uint32_t k0 = (uint32_t)a.seed, k1 = (uint32_t)(a.seed >> 32);

    u32x4 v[RPT];
    float w[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int64_t r = r0 + (t >> 4) + 16 * i;
        const uint16_t* row = nullptr;
        w[i] = 1.0f;
        if (r < a.rows) {
            if (a.src == nullptr) row = x + r * a.ld;
            else {
                const uint32_t choice = (uint32_t)a.src[r];
                if (choice < a.choices) {
                    row = x + (int64_t)(choice / a.top_k) * a.ld;
                    if (WEIGHTED) w[i] = a.weights[choice];
                }
            }
        }
        v[i] = row != nullptr && c < a.cols ? load8_start<STREAM>(row, c, a.cols) : u32x4{0u, 0u, 0u, 0u};
    }
    if (c < a.cols)
#pragma unroll
        for (int i = 0; i < RPT; ++i) v[i] = load8_end(v[i], c, a.cols);
    const bool ceil_rule = a.ceil_rule != 0;
    if (T) {
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int r = (t >> 4) + 16 * i;
            *reinterpret_cast<u32x4*>(&tile[r * 64 + (((t & 15) * 4 + 16 * (r / kRows)) & 63)]) = v[i];
            if (WEIGHTED && (t & 15) == 0) row_weight[r] = w[i];
        }
    }
    if (ROWS) {
        const MxOperand o = a.out;
        const int64_t block = c / kMxBlock;
        const bool inside = block * kMxBlock < a.cols;
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const int64_t r = r0 + (t >> 4) + 16 * i;
            uint32_t amax;
            float f[8];
            if (SR || WEIGHTED) widen8(v[i], f);
            if (WEIGHTED) {
                amax = 0u;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    f[j] = c + j < a.cols ? f[j] * w[i] : 0.0f;         // what a row lacks stays +0 under a negative weight
                    amax = max(amax, __float_as_uint(f[j]) & 0x7FFFFFFFu);
                }
            } else {
                uint32_t m = 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) m = pk_max_u16(m, v[i][j] & 0x7FFF7FFFu);
                amax = fold_max16(m) << 16;
            }
            amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
            amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
            const uint32_t byte = mx_scale_byte(amax, ceil_rule);
            uint32_t codes;
            if (SR) codes = mx_codes8_stochastic(f, byte, philox((uint32_t)(c >> 3), (uint32_t)r, z, 0u, k0, k1));
            else if (WEIGHTED) codes = mx_codes8_nearest(f, byte);
            else codes = mx_codes8_nearest(v[i], byte);
            if (r < a.rows && inside) {
                *reinterpret_cast<uint32_t*>(o.codes + z * o.batch + r * o.ld + (c >> 1)) = codes;
                if ((t & 3) == 0) o.scales[z * o.batch_s + r * o.ld_s + block] = (uint8_t)byte;
            }
        }
    }
    if (T) {
        const MxOperand o = a.out_t;
        __syncthreads();
        const int q = t & 3, pair = t >> 2;             // the lane's rows begin with q kRows
        const int64_t col = c0 + 2 * pair, row0 = r0 + q * kRows, block0 = row0 & ~31ll;
        uint32_t d[kRows];
#pragma unroll
        for (int j = 0; j < kRows; ++j) d[j] = tile[(kRows * q + j) * 64 + ((pair + 16 * q) & 63)];
        uint32_t m = 0u;
        float w_row[WEIGHTED ? kRows : 1];
        if (WEIGHTED) {
#pragma unroll
            for (int j = 0; j < kRows; ++j) w_row[j] = row_weight[kRows * q + j];
        } else {
#pragma unroll
            for (int j = 0; j < kRows; ++j) m = pk_max_u16(m, d[j] & 0x7FFF7FFFu);
        }
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            float f[kRows];
            uint32_t amax = side ? m & 0xFFFF0000u : m << 16;
            if (SR || WEIGHTED) {
#pragma unroll
                for (int j = 0; j < kRows; ++j) {
                    f[j] = __uint_as_float(side ? (d[j] & 0xFFFF0000u) : (d[j] << 16));
                    if (WEIGHTED) {
                        f[j] *= w_row[j];
                        amax = max(amax, __float_as_uint(f[j]) & 0x7FFFFFFFu);
                    }
                }
            }
            if (kRows == 8) {
                amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
                amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
            }
            const uint32_t byte = mx_scale_byte(amax, ceil_rule);
            uint32_t codes[kRows / 8];
#pragma unroll
            for (int g = 0; g < kRows / 8; ++g) {
                if (SR || WEIGHTED) {
                    float f8[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) f8[j] = f[8 * g + j];
                    if (SR) codes[g] = mx_codes8_stochastic(f8, byte, philox((uint32_t)(row0 >> 3) + g, (uint32_t)(col + side), z, 1u, k0, k1));
                    else codes[g] = mx_codes8_nearest(f8, byte);
                } else {
                    u32x4 p;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        p[j] = __builtin_amdgcn_perm(d[8 * g + 2 * j + 1], d[8 * g + 2 * j], side ? 0x07060302u : 0x05040100u);
                    codes[g] = mx_codes8_nearest(p, byte);
                }
            }
            if (col + side < a.cols && block0 < a.rows) {
                uint8_t* at = o.codes + z * o.batch + (col + side) * o.ld + (row0 >> 1);
                if constexpr (kRows == 32) *reinterpret_cast<u32x4*>(at) = u32x4{codes[0], codes[1], codes[2], codes[3]};
                else *reinterpret_cast<uint32_t*>(at) = codes[0];
                if (row0 == block0) o.scales[z * o.batch_s + (col + side) * o.ld_s + (block0 >> 5)] = (uint8_t)byte;
            }
        }
    }
}

// The rows form of tokens sorted by expert, rounded to nearest and without weights: every slot of a token holds the same codes.  So a
// token's row is read and quantised once and written to its choices' slots, and further workgroups, 32 slots each, fill the empty
// ones with zeros.  (8192 x 4096 into two slots each: 19 us = 5.4 TB/s of what is read and written once, 27 us on tokens that no
// cache holds; slot by slot, every row read and quantised twice, 30 us.)
constexpr int kFillSlots = 32;
template <int RPT>
__global__ __launch_bounds__(256) void k_mx_quantize_tokens(MxQuantArgs a, uint32_t col_tiles, uint32_t token_groups) {
    const int t = threadIdx.x;
    const MxOperand o = a.out;
    const uint32_t zero_byte = mx_scale_byte(0u, a.ceil_rule != 0);
    const int64_t blocks = (a.cols + kMxBlock - 1) / kMxBlock;
    if (blockIdx.x >= token_groups) {
        const int64_t slot0 = (int64_t)(blockIdx.x - token_groups) * kFillSlots + t / 64 * (kFillSlots / 4);
        for (int i = 0; i < kFillSlots / 4; ++i) {
            const int64_t slot = slot0 + i;
            if (slot >= a.rows || (uint32_t)a.src[slot] < a.choices) continue;
            for (int64_t b = t % 64; b < blocks; b += 64) {
                *reinterpret_cast<u32x4*>(o.codes + slot * o.ld + b * 16) = u32x4{0u, 0u, 0u, 0u};
                o.scales[slot * o.ld_s + b] = (uint8_t)zero_byte;
            }
        }
        return;
    }
    const uint32_t tile_id = tile_of(blockIdx.x, token_groups), ct = tile_id % col_tiles;
    const int64_t c = (int64_t)ct * kTileCols + (t & 15) * 8, block = c / kMxBlock;
    const int64_t token0 = (int64_t)(tile_id / col_tiles) * (RPT * 16) + (t >> 4);
    const uint32_t tokens = a.choices / a.top_k;
    constexpr uint32_t kAtOnce = 2;                     // slots on their way with the rows
    u32x4 v[RPT];
    uint32_t slots[RPT][kAtOnce];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int64_t token = token0 + 16 * i;
        v[i] = token < tokens && c < a.cols ? load8_start(a.x + token * a.ld, c, a.cols) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (uint32_t j = 0; j < kAtOnce; ++j)
            slots[i][j] = token < tokens && j < a.top_k ? (uint32_t)a.slot_of[token * a.top_k + j] : ~0u;
    }
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int64_t token = token0 + 16 * i;
        uint32_t m = 0u;
        if (c < a.cols) v[i] = load8_end(v[i], c, a.cols);
#pragma unroll
        for (int j = 0; j < 4; ++j) m = pk_max_u16(m, v[i][j] & 0x7FFF7FFFu);
        uint32_t amax = fold_max16(m) << 16;
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1));
        amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2));
        const uint32_t byte = mx_scale_byte(amax, a.ceil_rule != 0), codes = mx_codes8_nearest(v[i], byte);
        if (token >= tokens || block >= blocks) continue;
        auto put = [&](uint32_t slot) {
            if (slot >= (uint64_t)a.rows) return;
            *reinterpret_cast<uint32_t*>(o.codes + slot * o.ld + (c >> 1)) = codes;
            if ((t & 3) == 0) o.scales[slot * o.ld_s + block] = (uint8_t)byte;
        };
#pragma unroll
        for (uint32_t j = 0; j < kAtOnce; ++j) put(slots[i][j]);
        for (uint32_t j = kAtOnce; j < a.top_k; ++j) put((uint32_t)a.slot_of[token * a.top_k + j]);
    }
}

// Eight codes to eight BF16 values per lane, RPT rows of them; every value is exact.  Bound by the bytes written (14336 x 4096: 21.3 us =
// 6.9 TB/s).
template <int RPT, bool STREAM>
__global__ __launch_bounds__(256) void k_mx_dequantize(int64_t rows, int64_t cols, MxOperand op, uint16_t* y, int64_t ld_y, int64_t batch_y,
                                                       uint32_t col_tiles) {
    const uint32_t tile_id = tile_of(blockIdx.x, gridDim.x), ct = tile_id % col_tiles;
    const int64_t c = (int64_t)ct * kTileCols + (threadIdx.x & 15) * 8;
    const int64_t r0 = (int64_t)(tile_id / col_tiles) * (16 * RPT) + (threadIdx.x >> 4);
    const uint32_t z = blockIdx.z;
    if (c >= cols) return;
    uint32_t codes[RPT], byte[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int64_t r = min(r0 + 16 * i, rows - 1);
        codes[i] = *reinterpret_cast<const uint32_t*>(op.codes + z * op.batch + r * op.ld + (c >> 1));
        byte[i] = op.scales[z * op.batch_s + r * op.ld_s + (c >> 5)];
    }
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int64_t r = r0 + 16 * i;
        if (r >= rows) break;
        const float s = __uint_as_float(byte[i] << 23);     // the conversion reads the exponent field alone
        u32x4 out;
        out[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 0));
        out[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 1));
        out[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 2));
        out[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[i], s, 3));
        if (byte[i] == kMxNan) out = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        store8<STREAM>(y + (int64_t)z * batch_y + r * ld_y, c, cols, out);
    }
}

template <int RPT, bool ROWS, bool T, bool STREAM>
void quantize_form(const MxQuantArgs& a, uint32_t col_tiles, dim3 grid, hipStream_t st) {
    if (a.stochastic) {
        if (a.weights) k_mx_quantize<RPT, ROWS, T, true, true, false><<<grid, dim3(256), 0, st>>>(a, col_tiles);
        else k_mx_quantize<RPT, ROWS, T, true, false, STREAM><<<grid, dim3(256), 0, st>>>(a, col_tiles);
    } else {
        if (a.weights) k_mx_quantize<RPT, ROWS, T, false, true, false><<<grid, dim3(256), 0, st>>>(a, col_tiles);
        else k_mx_quantize<RPT, ROWS, T, false, false, STREAM><<<grid, dim3(256), 0, st>>>(a, col_tiles);
    }
}

}  // namespace

hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t st) {
    const uint32_t col_tiles = (uint32_t)((a.cols + kTileCols - 1) / kTileCols);
    const bool rows_form = a.out.codes != nullptr, t_form = a.out_t.codes != nullptr;
    const bool tall = a.rows * a.cols > kManyElements;
    // Tiles of 32 rows in the transposed form where those of 128 would be few, for which a lane's chain of work counts, not memory.  (Both
    // forms, nearest and stochastic, with tiles of 32 and of 128 rows: 1024 x 1024 3.6, 4.4 and 5.7, 8.7 us; 2048 x 4096 9.4, 13.1 and
    // 9.7, 14.9; 6144 x 4096 24.7, 31.9 and 22.0, 32.5; 14336 x 4096 58, 68 and 42, 62.)
    const bool short_t = t_form && (a.rows + 127) / 128 * col_tiles * a.batch <= (a.stochastic ? 1024 : 256);
    const int tile_rows = t_form ? short_t ? 32 : 128 : tall ? 32 : 16;
    if (a.src && !t_form && !a.weights && !a.stochastic) {
        const int64_t groups = ((int64_t)(a.choices / a.top_k) + tile_rows - 1) / tile_rows * col_tiles, fill = (a.rows + kFillSlots - 1) / kFillSlots;
        if (groups + fill > 0x7FFFFFFFll) return hipErrorInvalidValue;
        const dim3 grid((uint32_t)(groups + fill));
        if (tall) k_mx_quantize_tokens<2><<<grid, dim3(256), 0, st>>>(a, col_tiles, (uint32_t)groups);
        else k_mx_quantize_tokens<1><<<grid, dim3(256), 0, st>>>(a, col_tiles, (uint32_t)groups);
        return hipGetLastError();
    }
    const int64_t tiles = ((a.rows + tile_rows - 1) / tile_rows) * col_tiles;
    if (tiles > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)tiles, 1, (uint32_t)a.batch);
    // rows gathered by expert are read several times; the rows form alone is no faster past the caches (19.1 us against 19.7)
    const bool stream = t_form && a.src == nullptr && mx_streamed(a.rows * a.cols * a.batch, a.x, a.ld, a.batch_x, kMxStreamReadBytes);
    if (!t_form && tall) quantize_form<2, true, false, false>(a, col_tiles, grid, st);
    else if (!t_form) quantize_form<1, true, false, false>(a, col_tiles, grid, st);
    else if (short_t && rows_form) quantize_form<2, true, true, false>(a, col_tiles, grid, st);
    else if (short_t) quantize_form<2, false, true, false>(a, col_tiles, grid, st);
    else if (rows_form && stream) quantize_form<8, true, true, true>(a, col_tiles, grid, st);
    else if (rows_form) quantize_form<8, true, true, false>(a, col_tiles, grid, st);
    else if (stream) quantize_form<8, false, true, true>(a, col_tiles, grid, st);
    else quantize_form<8, false, true, false>(a, col_tiles, grid, st);
    return hipGetLastError();
}

hipError_t launch_mx_dequantize(int64_t rows, int64_t cols, int64_t batch, const MxOperand& op, uint16_t* y, int64_t ld_y, int64_t batch_y,
                                hipStream_t st) {
    const uint32_t col_tiles = (uint32_t)((cols + kTileCols - 1) / kTileCols);
    const bool tall = rows * cols * batch > kManyElements;
    const int tile_rows = tall ? 32 : 16;
    const int64_t tiles = ((rows + tile_rows - 1) / tile_rows) * col_tiles;
    if (tiles > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)tiles, 1, (uint32_t)batch);
    if (mx_streamed(rows * cols * batch, y, ld_y, batch_y)) k_mx_dequantize<2, true><<<grid, dim3(256), 0, st>>>(rows, cols, op, y, ld_y, batch_y, col_tiles);
    else if (tall) k_mx_dequantize<2, false><<<grid, dim3(256), 0, st>>>(rows, cols, op, y, ld_y, batch_y, col_tiles);
    else k_mx_dequantize<1, false><<<grid, dim3(256), 0, st>>>(rows, cols, op, y, ld_y, batch_y, col_tiles);
    return hipGetLastError();
}

}  // namespace mor
