// Products of microscaled 4-bit operands on the matrix cores.
#include <algorithm>

#include "mx_device.h"
#include "mx_launch.h"

namespace mor {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// One v_mfma_scale_f32_16x16x128_f8f6f4 with both operands in E2M1.  Lane l holds, of operand row l % 16, the 32 codes of
// block l / 16 (16 bytes) and that block's scale byte; of the result, rows 4 (l / 16) .. + 3 of the first operand in column
// l % 16, a row of the second.
__device__ __forceinline__ f32x4 mfma_mx(u32x4 a, uint32_t scale_a, u32x4 b, uint32_t scale_b, f32x4 c) {
    // the instruction reads the lower halves of the 32 bytes that other element types take
    const u32x8 va = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1), vb = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, va), __builtin_bit_cast(i32x8, vb), c, 4, 4, 0, (int)scale_a, 0,
                                                            (int)scale_b);
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

__device__ __forceinline__ u32x2 narrow4(const f32x4& v) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    const bf16x2 low = __builtin_convertvector((f32x2_t{v[0], v[1]}), bf16x2), high = __builtin_convertvector((f32x2_t{v[2], v[3]}), bf16x2);
    return u32x2{__builtin_bit_cast(uint32_t, low), __builtin_bit_cast(uint32_t, high)};
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
            const u32x2 w = narrow4(v);
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
            for (int j = 0; j < 4; ++j) acc[i][j] = mfma_mx(bv[j], bsv[j], av[i], as[i], acc[i][j]);
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

// ---- tiles through LDS -----------------------------------------------------------------------------------------------
//
// A workgroup of four waves forms BM x BN elements of C, each wave a quarter.  A stage is 128 of the depth, two 32 x 32 x 64 matrix
// instructions deep: 64 bytes of codes and 4 of scales per row, loaded from global memory straight into one of four LDS buffers.
// While stage s is multiplied, its later fragments and the first ones of stage s + 1 are read from LDS into registers, stage
// s + 2 is on its way and stage s + 3 is requested into the buffer that stage s - 1 left; one barrier per stage.
//
// One wave per SIMD (its 128 x 128 sums take half of the registers): an instruction is issued every four cycles at best, a
// matrix instruction takes 32.  Everything else is therefore spread over the matrix instructions, a few behind each, where it
// costs nothing; behind one another the same instructions took as long as the products.
//
// The four 16-byte pieces of a row lie permuted: piece j of row r at j ^ (r / 2 % 4), so that eight rows' pieces of the same
// depth, which one LDS cycle serves, fall into different banks.  Rows beyond the operand's last lie outside the buffer
// resource's range and arrive as zeros; so do the pieces behind a row's last block, whose lanes request an address out of range
// in the last stage, and stages beyond the last, whose range is empty.  The scale bytes behind the last block, loaded four at
// a time, are replaced by 2^0: whatever they hold, a NaN too, counts for nothing.

constexpr uint32_t kNowhere = 0x7FFFFFFFu;              // an offset that no range contains

// Bytes `first` .. `row_bytes` - 1 of an operand's rows row0 .. row0 + rows - 1, advancing along the rows.  The same in every lane:
// kept in scalar registers.
struct RowsBuffer {
    const uint8_t* base;
    int bytes;
    __device__ __forceinline__ RowsBuffer(const uint8_t* p, int64_t ld, int64_t row0, int64_t rows, int64_t first, int64_t row_bytes) {
        const uint64_t at = reinterpret_cast<uint64_t>(p + row0 * ld + first);
        // (the halves come back as signed numbers: widened as they are, a low half from 2^31 on would spill into the high one)
        const uint32_t low = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at), high = (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
        base = reinterpret_cast<const uint8_t*>(((uint64_t)high << 32) | low);
        bytes = __builtin_amdgcn_readfirstlane(rows > 0 && row_bytes > first ? (int)((rows - 1) * ld + row_bytes - first) : 0);
    }
    // The buffer resource from byte `step` of every row on.
    __device__ __forceinline__ u32x4 at(int step, bool exists) const {
        const uint64_t p = reinterpret_cast<uint64_t>(base) + step;
        return u32x4{(uint32_t)p, (uint32_t)(p >> 32) & 0xFFFFu, exists ? (uint32_t)max(bytes - step, 0) : 0u, 0x00020000u};
    }
};

// 16 bytes per lane from a buffer straight into LDS, one lane behind the other from `lds` on.  Written out because the compiler
// tracks the builtin's writes into LDS and, not being able to tell the four buffers apart across the loop, waits for all requests
// before it reads any buffer.  Nothing is loaded into registers here, and the waits stand in multiply_stage.  (M0 is a reserved
// register: the compiler sets it right before each use of its own, and nothing else in this kernel uses it.)
__device__ __forceinline__ void load_to_lds(uint8_t* lds, u32x4 buffer, uint32_t offset, int group_offset) {
    const uint32_t to = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 : : "s"(to), "v"(offset), "s"(buffer), "s"(group_offset) : "memory");
}

template <int BM, int BN>
struct TileShape {
    static constexpr int FM = BM / 64, FN = BN / 64;    // fragments of 32 rows of a wave
    static constexpr int kCodesB = BM * 64, kCodes = (BM + BN) * 64;            // bytes of a stage
    static constexpr int kScalesB = BM * 16, kScales = (BM + BN) * 16;          // bytes of four stages
    static constexpr int kRequests = kCodes / 4096, kScaleRequests = kScales / 4096;     // of one wave
};

// What a lane adds to the stage's base to request its pieces.
struct Request {
    RowsBuffer a, as, b, bs;
    uint32_t va, vb, vas, vbs;          // offset in the first group of rows
    uint32_t va_last, vb_last;          // the same in the last stage
    int step_a, step_b;                 // bytes between the groups of a wave
    int last;
};

// Wave w loads the codes of rows 16 (w + 4 i) .. + 15 of one stage: request `i` of A's, then B's.
template <int BM, int BN>
__device__ __forceinline__ void request_codes(uint8_t* lds, const Request& q, int stage, int wave, int i) {
    typedef TileShape<BM, BN> S;
    const bool exists = stage <= q.last;
    if (i < BM / 64) load_to_lds(lds + (wave + 4 * i) * 1024, q.a.at(stage * 64, exists), stage == q.last ? q.va_last : q.va, i * q.step_a);
    else load_to_lds(lds + S::kCodesB + (wave + 4 * (i - BM / 64)) * 1024, q.b.at(stage * 64, exists), stage == q.last ? q.vb_last : q.vb,
                     (i - BM / 64) * q.step_b);
}
// The scales of four stages, 16 bytes of a row: every row is a request of its own to the caches, so four stages share it.  Wave w
// loads those of rows 64 w .. + 63 of either operand, or of one of them where each has 128 rows.
template <int BM, int BN>
__device__ __forceinline__ void request_scales(uint8_t* lds, const Request& q, int stage, int wave) {
    typedef TileShape<BM, BN> S;
    static_assert(BM == BN && (BM == 256 || BM == 128), "which wave loads which rows");
    const bool exists = stage <= q.last;
    const u32x4 ra = q.as.at(stage * 4, exists), rb = q.bs.at(stage * 4, exists);
    if (BM == 256 || wave < 2) load_to_lds(lds + wave * 1024, ra, q.vas, 0);
    if (BM == 256) load_to_lds(lds + S::kScalesB + wave * 1024, rb, q.vbs, 0);
    else if (wave >= 2) load_to_lds(lds + wave * 1024, rb, q.vbs, 0);
}

// A lane's places in a buffer: its pieces of the two steps of a stage, its rows' scales.
struct Place {
    uint32_t a[2], b[2], sa, sb;
};

template <int FN>
struct Fragments {
    u32x4 a0, a1, b[FN];                // of a step: the first two of A, all of B
};
template <int FM, int FN>
struct Scales {
    u32x4 a[FM], b[FN];                 // word t: stage t of four; byte 0 for the first step, byte 2 for the second
};

// The scales of this lane's row: its block of a step is 0 or 1, so the words are shifted by `half` bytes.
__device__ __forceinline__ u32x4 own_scales(u32x4 d, uint32_t half) {
#pragma unroll
    for (int t = 0; t < 4; ++t) d[t] >>= 8 * half;
    return d;
}
// The last four stages: bytes of blocks from `blocks` on (counted from the first of these stages) become 2^0.
template <int FM, int FN>
__device__ __forceinline__ void mask_scales(Scales<FM, FN>& s, int blocks, uint32_t half) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        uint32_t keep = 0u;
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (t * 4 + b < blocks) keep |= 0xFFu << (8 * b);
        const uint32_t put = (0x7F7F7F7Fu & ~keep) >> (8 * half);
        keep >>= 8 * half;
#pragma unroll
        for (int i = 0; i < FM; ++i) s.a[i][t] = (s.a[i][t] & keep) | put;
#pragma unroll
        for (int j = 0; j < FN; ++j) s.b[j][t] = (s.b[j][t] & keep) | put;
    }
}

// c += b a^T with one v_mfma_scale_f32_32x32x64_f8f6f4, both operands in E2M1: lane l holds, of operand row l % 32, the 32 codes of
// block l / 32 and that block's scale, byte 2 STEP of a register; of the result, rows 8 (e / 4) + 4 (l / 32) + e % 4 of the first
// operand for its elements e in column l % 32, a row of the second.
//
// The compiler keeps the sums of a 128 x 128 wave in place only if told to: with the builtin it gives sums and addends different
// registers, which do not suffice (256 of 512 are sums), and moves them about.  As it does not look into the text, the two
// wait states between a vector instruction that writes an operand and a matrix instruction that reads it stand there, and
// settle() below stands before the first other use of the sums.
template <int STEP>
__device__ __forceinline__ void multiply(f32x16& c, u32x4 b, uint32_t sb, u32x4 a, uint32_t sa) {
    if (STEP == 0)
        asm("s_nop 1\n\tv_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
            : "+a"(c) : "v"(b), "v"(a), "v"(sb), "v"(sa));
    else
        asm("s_nop 1\n\tv_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4"
            : "+a"(c) : "v"(b), "v"(a), "v"(sb), "v"(sa));
}
// The last matrix instruction (eight passes of four cycles) has written its sums.
__device__ __forceinline__ void settle(f32x16& c) { asm volatile("s_nop 15\n\ts_nop 15" : "+a"(c)); }

// Half a stage, STEP of stage T of four: `cur` holds its first fragments; `next` receives those of the following step, from
// `lds_next`.  The requests of stage `stage` + 3 are spread over both steps; stage 0 requests the scales of the four stages after its
// own, stage 3 reads them.
template <int T, int STEP, int BM, int BN>
__device__ __forceinline__ void multiply_step(f32x16 (&acc)[BM / 64][BN / 64], const Fragments<BN / 64>& cur, Fragments<BN / 64>& next,
                                              const Scales<BM / 64, BN / 64>& scales, Scales<BM / 64, BN / 64>& fresh, const uint8_t* lds,
                                              const uint8_t* lds_next, uint8_t* lds_free, uint8_t* lds_scales, const Place& at, const Request& q,
                                              int stage, int wave, uint32_t half) {
    typedef TileShape<BM, BN> S;
    constexpr int FM = S::FM, FN = S::FN;
    static_assert(FM == FN, "one fragment of each operand is read per row of products");
    u32x4 a0 = cur.a0, a1 = cur.a1;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const u32x4 a = a0;
        a0 = a1;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            multiply<STEP>(acc[i][j], cur.b[j], scales.b[j][T], a, scales.a[i][T]);
            if (j == 0)
                a1 = *reinterpret_cast<const u32x4*>(i + 2 < FM ? lds + at.a[STEP] + (i + 2) * 2048 : lds_next + at.a[1 - STEP] + (i + 2 - FM) * 2048);
            if (j == 1) next.b[i] = *reinterpret_cast<const u32x4*>(lds_next + at.b[1 - STEP] + i * 2048);
            // this step's half of the requests, evenly over its products
            constexpr int kHalf = S::kRequests / 2;
#pragma unroll
            for (int r = 0; r < kHalf; ++r)
                if (i * FN + j == (r * FM * FN) / kHalf + FN / 2) request_codes<BM, BN>(lds_free, q, stage + 3, wave, STEP * kHalf + r);
            if (T == 0 && STEP == 1 && i == FM - 1 && j == FN - 1) request_scales<BM, BN>(lds_scales, q, stage + 4, wave);
            if (T == 3) {
                u32x4& f = STEP == 0 ? fresh.a[i] : fresh.b[i];
                if (j == 0) f = *reinterpret_cast<const u32x4*>(lds_scales + (STEP == 0 ? at.sa : at.sb) + i * 512);
                if (j == FN - 1) f = own_scales(f, half);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    next.a0 = a0;
    next.a1 = a1;
}

template <int T, int BM, int BN>
__device__ __forceinline__ void multiply_stage(f32x16 (&acc)[BM / 64][BN / 64], Fragments<BN / 64>& f0, Fragments<BN / 64>& f1,
                                               Scales<BM / 64, BN / 64>& scales, const uint8_t* lds, const uint8_t* lds_next, uint8_t* lds_free,
                                               uint8_t* lds_scales, const Place& at, const Request& q, int stage, int wave, uint32_t half,
                                               int blocks) {
    typedef TileShape<BM, BN> S;
    Scales<S::FM, S::FN> fresh;
    __builtin_amdgcn_s_waitcnt(0x0F70 | (S::kRequests + (T == 1 ? S::kScaleRequests : 0)));     // all but the latest stage's requests are here
    __syncthreads();
    multiply_step<T, 0, BM, BN>(acc, f0, f1, scales, fresh, lds, lds, lds_free, lds_scales, at, q, stage, wave, half);
    multiply_step<T, 1, BM, BN>(acc, f1, f0, scales, fresh, lds, lds_next, lds_free, lds_scales, at, q, stage, wave, half);
    if (T == 3) {
        scales = fresh;
        if (stage + 4 >= q.last) mask_scales(scales, blocks - (stage + 1) * 4, half);
    }
}

// A wave's sums to C by way of its LDS buffer, so that every row is written in pieces of 16 neighbouring bytes per lane: the
// accumulators hold 4 columns of 32 rows.  `kCols` columns at a time; pieces lie permuted by the row against bank conflicts.
template <bool F32, int FM, int FN>
__device__ __forceinline__ void store_tile(const MxProductArgs& p, uint8_t* lds, f32x16 (&acc)[FM][FN], int64_t base, int64_t m0, int64_t m_end,
                                           int64_t n0, int lane) {
    constexpr int kSize = F32 ? 4 : 2;
    constexpr int kCols = FN * 32 * kSize > 256 ? 256 / kSize : FN * 32;        // a row of up to 256 bytes
    constexpr int kRow = kCols * kSize, kPieces = kRow / 16, kLanes = 64 / kPieces;
    const int row = lane & 31, half = lane >> 5;
#pragma unroll
    for (int c0 = 0; c0 < FN * 32; c0 += kCols) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < kCols / 32; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x16 sums = acc[i][c0 / 32 + j];
                    const f32x4 v = {sums[4 * e], sums[4 * e + 1], sums[4 * e + 2], sums[4 * e + 3]};
                    uint8_t* at = lds + (32 * i + row) * kRow;
                    if (F32) *reinterpret_cast<f32x4*>(at + ((8 * j + 2 * e + half) ^ (row & (kPieces - 1))) * 16) = v;
                    else *reinterpret_cast<u32x2*>(at + ((4 * j + e) ^ (row & (kPieces - 1))) * 16 + half * 8) = narrow4(v);
                }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int piece = lane % kPieces;
        const int64_t n = n0 + c0 + piece * (16 / kSize);
#pragma unroll 4
        for (int r = lane / kPieces; r < FM * 32; r += kLanes) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(lds + r * kRow + (piece ^ (r & (kPieces - 1))) * 16);
            if (m0 + r >= m_end || n >= p.n) break;
            uint8_t* c = reinterpret_cast<uint8_t*>(p.c) + (base + (m0 + r) * p.ldc + n) * kSize;
            if (n + 16 / kSize <= p.n) __builtin_memcpy(c, &v, 16);
            else {
#pragma unroll 1
                for (int e = 0; n + e < p.n; ++e)       // the last columns
                    __builtin_memcpy(c + e * kSize, lds + r * kRow + (piece ^ (r & (kPieces - 1))) * 16 + e * kSize, kSize);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <int MODE, bool F32, int BM, int BN>
__global__ __launch_bounds__(256, 1) void k_mx_tile(MxProductArgs p, uint32_t m_tiles, uint32_t n_tiles) {
    typedef TileShape<BM, BN> S;
    constexpr int FM = S::FM, FN = S::FN;
    __shared__ __align__(1024) uint8_t buf0[S::kCodes];
    __shared__ __align__(1024) uint8_t buf1[S::kCodes];
    __shared__ __align__(1024) uint8_t buf2[S::kCodes];
    __shared__ __align__(1024) uint8_t buf3[S::kCodes];
    __shared__ __align__(1024) uint8_t buf_scales[S::kScales];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the eight XCDs in turn; each XCD takes a run of tiles, in patches of 8 tile rows, so that the tiles at work
    // together share their operands in its L2.
    uint32_t id = blockIdx.x;
    {
        const uint32_t total = gridDim.x, each = total / 8, more = total % 8, x = id % 8;
        id = x * each + min(x, more) + id / 8;
    }
    uint32_t z = 0;
    if (MODE == kMxDepth) { z = id / (m_tiles * n_tiles); id -= z * (m_tiles * n_tiles); }
    const uint32_t patch = id / (8 * n_tiles), in_patch = id - patch * (8 * n_tiles);
    const uint32_t tall = min(8u, m_tiles - patch * 8);
    const uint32_t m_tile = patch * 8 + in_patch % tall, n_tile = in_patch / tall;
    Tile t;
    if (!find_tile<MODE>(p, m_tile, z, BM, &t)) return;
    const int64_t n0 = (int64_t)n_tile * BN;
    const int blocks = __builtin_amdgcn_readfirstlane(t.k_end - t.k0);
    const int stages = (blocks + 3) / 4;

    const int64_t row_bytes = (int64_t)p.blocks * 16, row_scales = ((int64_t)p.blocks + 3) & ~3ll;
    const int64_t rows_a = min((int64_t)BM, t.m_end - t.m0), rows_b = min((int64_t)BN, p.n - n0);
    const int64_t of_b = MODE == kMxRows ? t.expert * p.batch_b : 0, of_bs = MODE == kMxRows ? t.expert * p.batch_bs : 0;
    const int piece = (lane & 3) ^ (lane >> 3 & 3);     // of row lane / 4 of a group
    const bool piece_in = (stages - 1) * 4 + piece < blocks;
    Request q{RowsBuffer(p.a, p.lda, t.m0, rows_a, (int64_t)t.k0 * 16, row_bytes), RowsBuffer(p.as, p.lda_s, t.m0, rows_a, t.k0, row_scales),
              RowsBuffer(p.b + of_b, p.ldb, n0, rows_b, (int64_t)t.k0 * 16, row_bytes),
              RowsBuffer(p.bs + of_bs, p.ldb_s, n0, rows_b, t.k0, row_scales),
              (uint32_t)(wave * 16 + (lane >> 2)) * (uint32_t)p.lda + piece * 16, (uint32_t)(wave * 16 + (lane >> 2)) * (uint32_t)p.ldb + piece * 16,
              (uint32_t)(wave * 64 + lane) * (uint32_t)p.lda_s, (uint32_t)((BM == 128 ? wave - 2 : wave) * 64 + lane) * (uint32_t)p.ldb_s, 0u, 0u,
              (int)p.lda * 64, (int)p.ldb * 64, stages - 1};
    q.va_last = piece_in ? q.va : kNowhere;
    q.vb_last = piece_in ? q.vb : kNowhere;

    const int row = lane & 31;
    const uint32_t half = lane >> 5;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    const uint32_t piece0 = (half ^ (row >> 1 & 3)) * 16, piece1 = ((half + 2) ^ (row >> 1 & 3)) * 16;
    const uint32_t row_a = (wm + row) * 64, row_b = S::kCodesB + (wn + row) * 64;
    const Place at{{row_a + piece0, row_a + piece1}, {row_b + piece0, row_b + piece1}, (uint32_t)(wm + row) * 16,
                   (uint32_t)S::kScalesB + (wn + row) * 16};

    f32x16 acc[FM][FN] = {};
    if (stages > 0) {
        Fragments<FN> f0, f1;
        Scales<FM, FN> sc;
        request_scales<BM, BN>(buf_scales, q, 0, wave);
#pragma unroll
        for (int i = 0; i < S::kRequests; ++i) request_codes<BM, BN>(buf0, q, 0, wave, i);
#pragma unroll
        for (int i = 0; i < S::kRequests; ++i) request_codes<BM, BN>(buf1, q, 1, wave, i);
#pragma unroll
        for (int i = 0; i < S::kRequests; ++i) request_codes<BM, BN>(buf2, q, 2, wave, i);
        __builtin_amdgcn_s_waitcnt(0x0F70 | (2 * S::kRequests & 15) | (2 * S::kRequests >> 4 << 14));
        __syncthreads();
        f0.a0 = *reinterpret_cast<const u32x4*>(buf0 + at.a[0]);
        f0.a1 = *reinterpret_cast<const u32x4*>(buf0 + at.a[0] + 2048);
#pragma unroll
        for (int j = 0; j < FN; ++j) f0.b[j] = *reinterpret_cast<const u32x4*>(buf0 + at.b[0] + j * 2048);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            sc.a[i] = own_scales(*reinterpret_cast<const u32x4*>(buf_scales + at.sa + i * 512), half);
            sc.b[i] = own_scales(*reinterpret_cast<const u32x4*>(buf_scales + at.sb + i * 512), half);
        }
        if (stages <= 4) mask_scales(sc, blocks, half);
        // (One way out of the loop: with more the compiler moves accumulators between registers.)
        for (int s = 0; s < stages; s += 4) {
            multiply_stage<0, BM, BN>(acc, f0, f1, sc, buf0, buf1, buf3, buf_scales, at, q, s, wave, half, blocks);
            if (s + 1 < stages) multiply_stage<1, BM, BN>(acc, f0, f1, sc, buf1, buf2, buf0, buf_scales, at, q, s + 1, wave, half, blocks);
            if (s + 2 < stages) multiply_stage<2, BM, BN>(acc, f0, f1, sc, buf2, buf3, buf1, buf_scales, at, q, s + 2, wave, half, blocks);
            if (s + 3 < stages) multiply_stage<3, BM, BN>(acc, f0, f1, sc, buf3, buf0, buf2, buf_scales, at, q, s + 3, wave, half, blocks);
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);             // the empty requests too, before the buffers are written
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) settle(acc[i][j]);
    __syncthreads();
    uint8_t* mine = wave == 0 ? buf0 : wave == 1 ? buf1 : wave == 2 ? buf2 : buf3;
    const int64_t base = MODE == kMxDepth ? t.expert * p.batch_c : 0;
    store_tile<F32, FM, FN>(p, mine, acc, base, t.m0 + wm, t.m_end, n0 + wn, lane);
}

}  // namespace

size_t mx_product_workspace(int64_t, int64_t, int64_t) { return 0; }

template <bool F32, int BM, int BN>
static hipError_t launch_tiles(int mode, const MxProductArgs& p, hipStream_t st) {
    const int64_t n_tiles = (p.n + BN - 1) / BN;
    int64_t m_tiles = (p.m + BM - 1) / BM;
    if (mode == kMxRows) m_tiles = p.m / BM + std::min<int64_t>(p.n_experts, p.m);
    const int64_t total = n_tiles * m_tiles * (mode == kMxDepth ? p.n_experts : 1);
    if (total > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)total);
    if (mode == kMxDense) k_mx_tile<kMxDense, F32, BM, BN><<<grid, dim3(256), 0, st>>>(p, (uint32_t)m_tiles, (uint32_t)n_tiles);
    else if (mode == kMxRows) k_mx_tile<kMxRows, F32, BM, BN><<<grid, dim3(256), 0, st>>>(p, (uint32_t)m_tiles, (uint32_t)n_tiles);
    else k_mx_tile<kMxDepth, F32, BM, BN><<<grid, dim3(256), 0, st>>>(p, (uint32_t)m_tiles, (uint32_t)n_tiles);
    return hipGetLastError();
}

hipError_t launch_mx_product(int mode, const MxProductArgs& p, void*, hipStream_t st) {
    // a tile's rows are addressed with 32-bit offsets
    const bool near = 256 * std::max(std::max(p.lda, p.ldb), std::max(p.lda_s, p.ldb_s)) < 0x7FFFFFFFll;
    if (near && p.m > 128) return p.f32 ? launch_tiles<true, 256, 256>(mode, p, st) : launch_tiles<false, 256, 256>(mode, p, st);
    if (near && p.m > 32) return p.f32 ? launch_tiles<true, 128, 128>(mode, p, st) : launch_tiles<false, 128, 128>(mode, p, st);
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
