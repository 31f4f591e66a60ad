// Products of microscaled 4-bit operands on the matrix cores.
#include <algorithm>

#include "mx_device.h"
#include "mx_launch.h"

namespace mor {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// One v_mfma_scale_f32_16x16x128_f8f6f4 with both operands in E2M1.  Lane l holds, of operand row l % 16, the 32 codes of
// block l / 16 (16 bytes) and that block's scale byte; of the result, rows 4 (l / 16) .. + 3 of the first operand in column
// l % 16, a row of the second.
template <int SA, int SB>
__device__ __forceinline__ f32x4 mfma_mx(const u32x4& a, uint32_t scale_a, const u32x4& b, uint32_t scale_b, const f32x4& c) {
    const i32x8 va = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 vb = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, SA, (int)scale_a, SB, (int)scale_b);
}

// Segment of expert e, kept inside [0, limit].
__device__ __forceinline__ void segment(const int32_t* offsets, int e, int64_t limit, int64_t* lo, int64_t* hi) {
    const int64_t a = offsets[e], b = offsets[e + 1];
    *lo = a < 0 ? 0 : (a > limit ? limit : a);
    *hi = b < *lo ? *lo : (b > limit ? limit : b);
}

// What one workgroup's tile covers; false: nothing.
struct Tile {
    int64_t m0, m_end;                  // rows of A and C
    int32_t k0, k_end;                  // blocks of the depth
    int32_t expert;
};

// kMxRows: which expert's rows are tile `index`, if the segments are cut into tiles of `height` rows each.  Every wave finds it by
// itself: 64 experts at a time, a lane each, running sums of their tiles.
__device__ __forceinline__ bool find_rows(const MxProductArgs& p, uint32_t index, int height, Tile* tile) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0u;
    for (int e0 = 0; e0 < p.n_experts; e0 += 64) {
        int64_t lo = 0, hi = 0;
        if (e0 + lane < p.n_experts) segment(p.offsets, e0 + lane, p.m, &lo, &hi);
        const uint32_t tiles = (uint32_t)((hi - lo + height - 1) / height);
        uint32_t upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t other = (uint32_t)__shfl_up((int)upto, d);
            if (lane >= d) upto += other;
        }
        const uint64_t hit = __ballot(before + upto > index);
        if (hit) {
            const int who = __ffsll((unsigned long long)hit) - 1;
            const uint32_t first = before + (uint32_t)__shfl((int)(upto - tiles), who);
            const int64_t lo_w = ((int64_t)__shfl((int)(lo >> 32), who) << 32) | (uint32_t)__shfl((int)lo, who);
            const int64_t hi_w = ((int64_t)__shfl((int)(hi >> 32), who) << 32) | (uint32_t)__shfl((int)hi, who);
            tile->expert = e0 + who;
            tile->m0 = lo_w + (int64_t)(index - first) * height;
            tile->m_end = hi_w;
            return true;
        }
        before += (uint32_t)__shfl((int)upto, 63);
    }
    return false;
}

template <int MODE>
__device__ __forceinline__ bool find_tile(const MxProductArgs& p, uint32_t m_tile, uint32_t z, int height, Tile* tile) {
    tile->k0 = 0;
    tile->k_end = p.blocks;
    tile->expert = 0;
    if (MODE == kMxRows) return find_rows(p, m_tile, height, tile);
    tile->m0 = (int64_t)m_tile * height;
    tile->m_end = p.m;
    if (MODE == kMxDepth) {
        int64_t lo, hi;
        tile->expert = (int)z;
        segment(p.offsets, (int)z, (int64_t)p.blocks * kMxBlock, &lo, &hi);
        tile->k0 = (int32_t)(lo / 128 * 4);
        tile->k_end = (int32_t)((hi + kMxBlock - 1) / kMxBlock);
    }
    return true;
}

// Four consecutive elements of a row of C.
__device__ __forceinline__ void store4(const MxProductArgs& p, int64_t at, int64_t n, const f32x4& v) {
    if (p.f32) {
        float* c = reinterpret_cast<float*>(p.c) + at;
        if (n + 4 <= p.n) __builtin_memcpy(c, &v, 16);
        else
            for (int j = 0; j < 4; ++j)
                if (n + j < p.n) c[j] = v[j];
    } else {
        uint16_t* c = reinterpret_cast<uint16_t*>(p.c) + at;
        if (n + 4 <= p.n) {
            const u32x2 w{bf16_of(v[0]) | (bf16_of(v[1]) << 16), bf16_of(v[2]) | (bf16_of(v[3]) << 16)};
            __builtin_memcpy(c, &w, 8);
        }
        else
            for (int j = 0; j < 4; ++j)
                if (n + j < p.n) c[j] = (uint16_t)bf16_of(v[j]);
    }
}

// One wave: 32 rows of C x 64 columns, operands from global memory straight into registers.
constexpr int kWaveM = 32, kWaveN = 64;
template <int MODE>
__global__ __launch_bounds__(64) void k_mx_product(MxProductArgs p, uint32_t n_tiles) {
    const int lane = threadIdx.x;
    const uint32_t n_tile = blockIdx.x % n_tiles, m_tile = blockIdx.x / n_tiles;
    Tile t;
    if (!find_tile<MODE>(p, m_tile, blockIdx.z, kWaveM, &t)) return;
    const int64_t n0 = (int64_t)n_tile * kWaveN;
    const uint8_t* b = p.b + (MODE == kMxRows ? t.expert * p.batch_b : 0);
    const uint8_t* bs = p.bs + (MODE == kMxRows ? t.expert * p.batch_bs : 0);
    const int row = lane & 15, part = lane >> 4;
    f32x4 acc[2][4] = {};
    for (int32_t k = t.k0; k < t.k_end; k += 4) {
        const int32_t block = min(k + part, t.k_end - 1);
        const bool in = k + part < t.k_end;
        u32x4 av[2], bv[4];
        uint32_t as[2], bsv[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t r = min(t.m0 + 16 * i + row, t.m_end - 1);
            av[i] = *reinterpret_cast<const u32x4*>(p.a + r * p.lda + (int64_t)block * 16);
            as[i] = p.as[r * p.lda_s + block];
            if (!in) { av[i] = u32x4{0u, 0u, 0u, 0u}; as[i] = 127u; }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = min(n0 + 16 * i + row, p.n - 1);
            bv[i] = *reinterpret_cast<const u32x4*>(b + r * p.ldb + (int64_t)block * 16);
            bsv[i] = bs[r * p.ldb_s + block];
            if (!in) { bv[i] = u32x4{0u, 0u, 0u, 0u}; bsv[i] = 127u; }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = mfma_mx<0, 0>(bv[j], bsv[j], av[i], as[i], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t m = t.m0 + 16 * i + row;
        if (m >= t.m_end) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + 16 * j + 4 * part;
            if (n < p.n) store4(p, (MODE == kMxDepth ? t.expert * p.batch_c : 0) + m * p.ldc + n, n, acc[i][j]);
        }
    }
}

}  // namespace

size_t mx_product_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx_product(int mode, const MxProductArgs& p, void*, hipStream_t st) {
    const int64_t n_tiles = (p.n + kWaveN - 1) / kWaveN;
    int64_t m_tiles = (p.m + kWaveM - 1) / kWaveM;
    if (mode == kMxRows) m_tiles = p.m / kWaveM + std::min<int64_t>(p.n_experts, p.m);    // each segment ends in one part tile at most
    if (n_tiles * m_tiles > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)(n_tiles * m_tiles), 1, mode == kMxDepth ? (uint32_t)p.n_experts : 1u);
    if (mode == kMxDense) k_mx_product<kMxDense><<<grid, dim3(64), 0, st>>>(p, (uint32_t)n_tiles);
    else if (mode == kMxRows) k_mx_product<kMxRows><<<grid, dim3(64), 0, st>>>(p, (uint32_t)n_tiles);
    else k_mx_product<kMxDepth><<<grid, dim3(64), 0, st>>>(p, (uint32_t)n_tiles);
    return hipGetLastError();
}

}  // namespace mor
