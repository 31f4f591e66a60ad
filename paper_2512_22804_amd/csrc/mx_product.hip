// Products of microscaled 4-bit operands on the matrix cores.
#include <algorithm>
#include <cmath>
#include <type_traits>

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

// How many tiles that makes.
__device__ __forceinline__ uint32_t count_rows(const MxProductArgs& p, int height) {
    const int lane = threadIdx.x & 63;
    uint32_t tiles = 0u;
    for (int e = lane; e < p.n_experts; e += 64) {
        int64_t lo, hi;
        segment(p.offsets, e, p.m, &lo, &hi);
        tiles += (uint32_t)((hi - lo + height - 1) / height);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) tiles += (uint32_t)__shfl_xor((int)tiles, d);
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)tiles);
}

template <int MODE>
__device__ __forceinline__ bool find_tile(const MxProductArgs& p, uint32_t m_tile, uint32_t z, int height, Tile* tile) {
    tile->k0 = 0;
    tile->k_end = p.blocks;
    tile->expert = 0;
    if (MODE == kMxRows) return find_rows(p, m_tile, height, tile);
    tile->m0 = (int64_t)m_tile * height;
    tile->m_end = p.m;
    if (MODE == kMxDense && p.splits > 1) {             // z-th part of the depth, whole stages
        const int32_t each = ((p.blocks + 7) / 8 + p.splits - 1) / p.splits * 8;
        tile->k0 = min((int32_t)z * each, p.blocks);
        tile->k_end = min(tile->k0 + each, p.blocks);
        tile->expert = (int)z;
    }
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

// One wave: 32 rows of C x 64 columns, operands from global memory straight into registers.  For operands whose rows are too far
// apart for the kernels below (2^31 bytes and more between 256 of them).
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
// A workgroup of four waves forms BM x BN elements of C, each wave a quarter.  A stage is 256 of the depth: 128 bytes of codes and 8
// of scales per row, loaded from global memory straight into one of two LDS buffers.  Pieces of 128 bytes matter: the L2 serves a
// CU 57 bytes per cycle in whole lines, 30 in halves, which bound this kernel when a stage was 128 deep (8192 x 14336 x 4096:
// 274 us).
//
// A stage has four steps of 64, one 32 x 32 x 64 matrix instruction deep.  The fragments of a step are read from LDS into registers
// while the step before is multiplied.  Those of a stage's last step are thus in registers when it begins: there is the barrier, the
// next stage has arrived, and the one after it is requested into the buffer that is free now; it has four steps to arrive.
//
// With one wave per SIMD (its 128 x 128 sums take half of the registers) an instruction is issued every four cycles at best; a
// matrix instruction takes 32.  Everything else is therefore spread over the matrix instructions, a few behind each, where it
// costs nothing.
//
// The eight 16-byte pieces of a row lie permuted: piece j of row r at j ^ (r / 2 % 8).  One LDS cycle serves 16 lanes' pieces, of
// rows 0-3, 12-15, 20-23 and 24-27 of a fragment for example, which so fall into different banks.  Rows beyond the operand's last
// lie outside the buffer resource's range and arrive as zeros; so do the pieces behind a row's last block, whose lanes request an
// address out of range in the last stage, and stages beyond the last, whose range is empty.  The scale bytes behind the last
// block, loaded 16 at a time, are replaced by 2^0: whatever they hold, a NaN too, counts for nothing.
//
// 8192 x 14336 x 4096: 241 to 258 us on several cards, 3.7 to 4.0 PFLOP/s.  The same instructions on random operands that stay in registers
// reach 6.4 at 1.65 GHz, the clock that the power allows, and 9.6 on zeros.  Here the matrix instructions are busy for 49 % of the
// cycles and LDS for 20 %.  A tile's way out (its sums through LDS to memory, about 8 us of 35) is not covered by the next one's
// products, since the sums and their successors do not both fit into the registers; the rest goes in the stages, between the
// matrix instructions.

constexpr uint32_t kNowhere = 0x7FFFFFFFu;              // an offset that no range contains

// Bytes `first` .. `row_bytes` - 1 of an operand's rows row0 .. row0 + rows - 1, advancing along the rows.  The same in every lane:
// kept in scalar registers.
struct RowsBuffer {
    const uint8_t* base;
    int bytes;
    RowsBuffer() = default;
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
// before it reads any buffer.  Nothing is loaded into registers here, and the waits stand in take_tiles.  (M0 is a reserved
// register: the compiler sets it right before each use of its own, and nothing else in this kernel uses it.)  Nor does the compiler
// look into the text for wait states: five must lie between a vector instruction that writes a scalar register (v_readfirstlane, or
// v_readlane where one was spilled) and a buffer load that reads it, so they stand here, whatever comes before.
__device__ __forceinline__ void load_to_lds(uint32_t lds, u32x4 buffer, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(offset), "s"(buffer) : "memory");
}

template <int BM, int BN>
struct TileShape {
    static constexpr int FM = BM / 64, FN = BN / 64;    // fragments of 32 rows of a wave
    static constexpr int kCodesB = BM * 128, kCodes = (BM + BN) * 128;          // bytes of a stage
    static constexpr int kScalesB = BM * 16, kScales = (BM + BN) * 16;          // bytes of two stages
    static constexpr int kRequests = kCodes / 4096, kFirstRequests = (kRequests + 1) / 2;       // of one wave
    static constexpr int kScalesAt = 2 * kCodes, kLds = kScalesAt + 2 * kScales;
};

// What a lane adds to the stage's base to request its pieces.
struct Request {
    RowsBuffer a, as, b, bs;
    uint32_t va, vb, vas, vbs;          // offset in the first group of rows
    uint32_t va_last, vb_last;          // the same in the last stage
    int step_a, step_b;                 // bytes between the groups of a wave
    int last;
};

// Wave w loads the codes of rows 8 (w + 4 i) .. + 7 of one stage: request `i` of A's, then B's.
struct Asked {
    u32x4 buffer;
    uint32_t lds, offset;
};
template <class S>
__device__ __forceinline__ Asked codes_request(uint32_t lds, const Request& q, int stage, int wave, int i) {
    constexpr int kOfA = S::kCodesB / 4096;
    const bool exists = stage <= q.last;
    if (i < kOfA) return {q.a.at(stage * 128, exists), lds + (wave + 4 * i) * 1024, (stage == q.last ? q.va_last : q.va) + i * q.step_a};
    return {q.b.at(stage * 128, exists), lds + S::kCodesB + (wave + 4 * (i - kOfA)) * 1024, (stage == q.last ? q.vb_last : q.vb) + (i - kOfA) * q.step_b};
}
template <class S>
__device__ __forceinline__ void request_codes(uint32_t lds, const Request& q, int stage, int wave, int i) {
    const Asked r = codes_request<S>(lds, q, stage, wave, i);
    load_to_lds(r.lds, r.buffer, r.offset);
}
// The scales of two stages, 16 bytes of a row.  Wave w loads those of rows 64 w .. + 63 of either operand; where one has fewer, several
// waves load the same.
template <class S>
__device__ __forceinline__ void request_scales(uint32_t lds, const Request& q, int stage, int wave) {
    const bool exists = stage <= q.last;
    load_to_lds(lds + wave % (S::kScalesB / 1024) * 1024, q.as.at(stage * 8, exists), q.vas);
    load_to_lds(lds + S::kScalesB + wave % ((S::kScales - S::kScalesB) / 1024) * 1024, q.bs.at(stage * 8, exists), q.vbs);
}

// A lane's places in a buffer: its pieces of the four steps of a stage, its rows' scales.
struct Place {
    uint32_t a[4], b[4], sa, sb;
};

template <int FM, int FN>
struct Fragments {
    u32x4 a[FM], b[FN];
};
template <int FM, int FN>
struct Scales {
    u32x2 a[FM], b[FN];                 // of a stage; bytes 0 and 2 of a word: two steps
};
template <int FM, int FN>
__device__ __forceinline__ void read_fragments(Fragments<FM, FN>& f, const uint8_t* lds, const Place& at, int step) {
#pragma unroll
    for (int i = 0; i < FM; ++i) f.a[i] = *reinterpret_cast<const u32x4*>(lds + at.a[step] + i * 4096);
#pragma unroll
    for (int j = 0; j < FN; ++j) f.b[j] = *reinterpret_cast<const u32x4*>(lds + at.b[step] + j * 4096);
}

// The scales of this lane's row: its block of a step is 0 or 1, so the words are shifted by `half` bytes; `keep` and `put` replace what
// lies behind the last block.
struct ScaleMask {
    u32x2 keep, put;
    uint32_t shift;
    // `blocks`: those that the stage has, 8 or more: all
    __device__ __forceinline__ ScaleMask(int blocks, uint32_t half) {
        shift = 8 * half;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int n = min(max(blocks - 4 * t, 0), 4);
            const uint32_t in = n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
            keep[t] = in >> shift;
            put[t] = (0x7F7F7F7Fu & ~in) >> shift;
        }
    }
    __device__ __forceinline__ u32x2 operator()(u32x2 d) const {
        return u32x2{((d[0] >> shift) & keep[0]) | put[0], ((d[1] >> shift) & keep[1]) | put[1]};
    }
};

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
// The same and load_to_lds behind it.  The matrix instruction and the states before it are four of the five that the request wants
// (8192 x 14336 x 4096: 247 us, as long as with two states before each request; 250 with five in a text of their own).
template <int STEP>
__device__ __forceinline__ void multiply_and_request(f32x16& c, u32x4 b, uint32_t sb, u32x4 a, uint32_t sa, const Asked& r) {
    if (STEP == 0)
        asm volatile("s_mov_b32 m0, %5\n\ts_nop 2\n\t"
                     "v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4\n\t"
                     "buffer_load_dwordx4 %6, %7, 0 offen lds"
                     : "+a"(c) : "v"(b), "v"(a), "v"(sb), "v"(sa), "s"(r.lds), "v"(r.offset), "s"(r.buffer) : "memory");
    else
        asm volatile("s_mov_b32 m0, %5\n\ts_nop 2\n\t"
                     "v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4\n\t"
                     "buffer_load_dwordx4 %6, %7, 0 offen lds"
                     : "+a"(c) : "v"(b), "v"(a), "v"(sb), "v"(sa), "s"(r.lds), "v"(r.offset), "s"(r.buffer) : "memory");
}
// Before the first other use of the sums: the last matrix instruction (eight passes of four cycles) has written its own.
template <int FM, int FN>
__device__ __forceinline__ void settle(f32x16 (&acc)[FM][FN]) {
    asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc[FM - 1][FN - 1]));
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) asm volatile("" : "+a"(acc[i][j]));
}

// Step STEP of a stage: multiplies `cur` and reads `next` from `next_a`, `next_b` (this lane's pieces there), both in slots, one behind
// each matrix instruction.  From the last step on the requests of stage `ahead` into `to`: a CU takes one of its waves' requests
// every 16 cycles, and a wave that has to wait with one cannot go on with its products either: half of them go into the
// first step of the next stage (512 x 4096 x 14336: 80 us; all in the last step 88, over three steps 81, over four 92).  In the
// last step also the scales of the next stage.
template <int STEP, class S>
__device__ __forceinline__ void multiply_step(f32x16 (&acc)[S::FM][S::FN], const Fragments<S::FM, S::FN>& cur, Fragments<S::FM, S::FN>& next,
                                              const Scales<S::FM, S::FN>& scales, Scales<S::FM, S::FN>& fresh, const uint8_t* next_a,
                                              const uint8_t* next_b, const uint8_t* scales_a, const uint8_t* scales_b, uint32_t to,
                                              const Request& q, int ahead, int wave, const ScaleMask& mask) {
    constexpr int FM = S::FM, FN = S::FN, kSlots = FM * FN, kWord = STEP / 2;
    constexpr int kFirst = S::kFirstRequests, kFrom = STEP == 3 ? 0 : kFirst;
    constexpr int kCount = STEP == 3 ? kFirst : STEP == 0 ? S::kRequests - kFirst : 0;
    static_assert(kCount <= kSlots, "one request behind a matrix instruction");
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int slot = i * FN + j;
            int asked = -1;                             // at most one request behind a matrix instruction
#pragma unroll
            for (int r = 0; r < kCount; ++r)
                if (slot == r * kSlots / (kCount ? kCount : 1)) asked = r;
            if (asked < 0) multiply<STEP % 2>(acc[i][j], cur.b[j], scales.b[j][kWord], cur.a[i], scales.a[i][kWord]);
            else multiply_and_request<STEP % 2>(acc[i][j], cur.b[j], scales.b[j][kWord], cur.a[i], scales.a[i][kWord],
                                                codes_request<S>(to, q, ahead, wave, kFrom + asked));
            // the reads over the first half of the slots, so that they are complete by the end
#pragma unroll
            for (int r = 0; r < FM + FN; ++r)
                if (slot == r * ((kSlots + 1) / 2) / (FM + FN)) {
                    if (r < FN) next.b[r] = *reinterpret_cast<const u32x4*>(next_b + r * 4096);
                    else next.a[r - FN] = *reinterpret_cast<const u32x4*>(next_a + (r - FN) * 4096);
                }
            if (STEP == 3) {
                if (j == 0) fresh.a[i] = *reinterpret_cast<const u32x2*>(scales_a + i * 512);
                if (i == 0) fresh.b[j] = *reinterpret_cast<const u32x2*>(scales_b + j * 512);
                if (j == FN - 1) fresh.a[i] = mask(fresh.a[i]);
                if (i == FM - 1) fresh.b[j] = mask(fresh.b[j]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// A wave's sums to C by way of its LDS buffer, so that every row is written in pieces of 16 neighbouring bytes per lane: the
// accumulators hold 4 columns of 32 rows.  `kCols` columns at a time; pieces lie permuted by the row against bank conflicts.
template <bool F32, int FM, int FN, int BYTES, bool DEPTH>
__device__ __forceinline__ void store_tile(const MxProductArgs& p, uint8_t* lds, f32x16 (&acc)[FM][FN], int64_t base, int64_t m0, int64_t m_end,
                                           int64_t n0, int lane, bool words) {
    constexpr int kSize = F32 ? 4 : 2;
    constexpr int kMost = BYTES / (FM * 32) >= 256 ? 256 : 128;                 // bytes of a row at a time
    constexpr int kCols = FN * 32 * kSize > kMost ? kMost / kSize : FN * 32;
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
        const int piece = lane % kPieces, first = lane / kPieces;
        const int64_t n = n0 + c0 + piece * (16 / kSize);
        const bool inside = n + 16 / kSize <= p.n;      // a whole piece
        if (words) {
            // Rows of 4-byte words: those from `m_end` on and pieces that are not whole lie outside the buffer, which ends with the last
            // row's last column; always the same number of stores.
            const int64_t rows = min(m_end - m0, (int64_t)FM * 32), columns = min((int64_t)kCols, max(p.n - n0 - c0, (int64_t)0));
            const uint32_t ld = (uint32_t)p.ldc * kSize;
            const BufRsrc out = make_buf_window(reinterpret_cast<uint8_t*>(p.c) + (base + m0 * p.ldc + n0 + c0) * kSize,
                                                rows > 0 ? (uint32_t)(rows - 1) * ld + (uint32_t)columns * kSize : 0u);
            const uint32_t start = inside ? first * ld + piece * 16 : kNowhere;     // (which 128 rows more do not bring back into range)
            const auto store_rows = [&](auto aux) {
                uint32_t at = start;
#pragma unroll
                for (int r = 0; r < FM * 32; r += kLanes) {
                    const int row_r = first + r;        // its swizzle repeats: kLanes divides kPieces or the other way round
                    buf_store16<decltype(aux)::value>(out, at, *reinterpret_cast<const u32x4*>(lds + row_r * kRow + (piece ^ (row_r & (kPieces - 1))) * 16));
                    at += kLanes * ld;
                }
            };
            // The experts' results, as large as their weights, go past the caches if their rows consist of whole lines (16 of 2048 x 4096:
            // 147 us, 170 through the caches; 60 of 442 x 1000, whose lines two waves write: 42 and 29).
            if (DEPTH && p.c_lines) store_rows(std::integral_constant<int, kBufStoreNt>{});
            else store_rows(std::integral_constant<int, 0>{});
        }
        if (n < p.n && !(words && inside)) {
#pragma unroll 1
            for (int r = first; r < FM * 32; r += kLanes) {
                if (m0 + r >= m_end) break;
                const uint8_t* v = lds + r * kRow + (piece ^ (r & (kPieces - 1))) * 16;
                uint8_t* c = reinterpret_cast<uint8_t*>(p.c) + (base + (m0 + r) * p.ldc + n) * kSize;
                if (inside) __builtin_memcpy(c, v, 16);
                else {
#pragma unroll 1
                    for (int e = 0; n + e < p.n; ++e) __builtin_memcpy(c + e * kSize, v + e * kSize, kSize);    // the last columns
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// A tile and what its requests need.
template <class S>
struct TileWork {
    Tile t;
    int64_t n0;
    int blocks, stages;
    Request q;
};

// Values that are the same in every lane, which the compiler cannot see where they come out of a search by all lanes.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t low = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), high = (uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)(((uint64_t)high << 32) | low);
}
__device__ __forceinline__ void make_uniform(RowsBuffer* b) {
    b->base = reinterpret_cast<const uint8_t*>(uniform((int64_t)reinterpret_cast<uintptr_t>(b->base)));
    b->bytes = uniform(b->bytes);
}
template <class S>
__device__ __forceinline__ void make_uniform(TileWork<S>* w) {
    make_uniform(&w->q.a);
    make_uniform(&w->q.as);
    make_uniform(&w->q.b);
    make_uniform(&w->q.bs);
    w->q.last = uniform(w->q.last);
    w->blocks = uniform(w->blocks);
    w->stages = uniform(w->stages);
    w->t.m0 = uniform(w->t.m0);
    w->t.m_end = uniform(w->t.m_end);
    w->t.expert = uniform(w->t.expert);
    w->n0 = uniform(w->n0);
}

// The tiles of a workgroup, one after the other.  The XCDs take the workgroups in turn; each gets a run of tiles, in patches of 8
// tile rows, so that the tiles at work together share their operands in its L2.  The experts' results, whose depths differ, are dealt
// out in shorter runs, an eighth of an expert's each: otherwise the XCD with the longest depths finishes last.
struct Walk {
    uint32_t left;                      // tiles (or pieces) of this workgroup's XCD from the present one on
    uint32_t z, patch, in_patch;        // expert or part, patch, tile in it
    uint32_t n_tiles, m_tiles, total;
    uint32_t x, first, stride;          // XCD, which of its workgroups this is, how many it has
    uint32_t run, in_run;               // tiles of a run, which one of them
    uint32_t mine;                      // tiles of this XCD
    __device__ __forceinline__ Walk(uint32_t all, uint32_t mt, uint32_t nt, bool shorter) {
        total = all; n_tiles = nt; m_tiles = mt;
        x = blockIdx.x % 8;
        first = blockIdx.x / 8;
        stride = (gridDim.x - x + 7) / 8;
        run = shorter ? max(mt * nt / 8, 1u) : ~0u;
        mine = total / 8 + (x < total % 8 ? 1u : 0u);
        if (shorter) {
            const uint32_t runs = total / run;
            mine = (runs / 8 + (x < runs % 8 ? 1u : 0u)) * run + (x == runs % 8 ? total - runs * run : 0u);
        }
    }
    // The XCD's tile number `at`.
    __device__ __forceinline__ void place(uint32_t at, bool many, bool shorter) {
        uint32_t id = x * (total / 8) + min(x, total % 8) + at;
        in_run = at;
        if (shorter) {
            in_run = at % run;
            id = (at / run * 8 + x) * run + in_run;
        }
        z = many ? id / (m_tiles * n_tiles) : 0u;
        id -= z * (m_tiles * n_tiles);
        patch = id / (8 * n_tiles);
        in_patch = id - patch * (8 * n_tiles);
    }
    __device__ __forceinline__ void next(bool many, bool shorter) {
        left = left > stride ? left - stride : 0u;
        in_patch += stride;
        if (shorter)
            for (in_run += stride; in_run >= run; in_run -= run) in_patch += 7 * run;    // the runs of the other XCDs
        for (;;) {                      // patches hold 8 n_tiles tiles, the last one of an expert fewer
            const uint32_t size = min(8u, m_tiles - patch * 8) * n_tiles;
            if (in_patch < size || !left) break;
            in_patch -= size;
            if (++patch * 8 >= m_tiles && many) { patch = 0; ++z; }
        }
    }
};

// What the walk's present tile needs, or piece `piece_of` of a tile of PIECES: 2, one above the other, or 4; false: nothing.
template <int MODE, int BM, int BN, int PIECES, class S>
__device__ __forceinline__ bool find_work(const MxProductArgs& p, const Walk& walk, uint32_t piece_of, int lane, int wave, TileWork<S>* w) {
    const uint32_t tall = min(8u, walk.m_tiles - walk.patch * 8), z = walk.z;
    uint32_t in_patch = walk.in_patch;
    const uint32_t n_tile = tall == 8 ? in_patch / 8 : in_patch / tall, m_tile = walk.patch * 8 + (in_patch - n_tile * tall);
    Tile& t = w->t;
    if (!find_tile<MODE>(p, m_tile, z, PIECES > 1 ? 2 * BM : BM, &t)) return false;
    w->n0 = (int64_t)n_tile * (PIECES == 4 ? 2 * BN : BN);
    if (PIECES > 1) {
        t.m0 += (piece_of & 1) * BM;
        w->n0 += (piece_of >> 1) * BN;
        if (!__builtin_amdgcn_readfirstlane(t.m0 < t.m_end && w->n0 < p.n)) return false;
    }
    w->blocks = __builtin_amdgcn_readfirstlane(t.k_end - t.k0);
    w->stages = max((w->blocks + 7) / 8, 1);             // (no depth at all: one stage of zeros)
    const int64_t row_bytes = (int64_t)p.blocks * 16, row_scales = ((int64_t)p.blocks + 3) & ~3ll;
    const int64_t rows_a = min((int64_t)BM, t.m_end - t.m0), rows_b = min((int64_t)BN, p.n - w->n0);
    const int64_t of_b = MODE == kMxRows ? t.expert * p.batch_b : 0, of_bs = MODE == kMxRows ? t.expert * p.batch_bs : 0;
    const int piece = (lane & 7) ^ ((lane >> 4) + 4 * (wave & 1));      // of row lane / 8 of a group of 8
    const bool piece_in = (w->stages - 1) * 8 + piece < w->blocks;
    Request& q = w->q;
    q.a = RowsBuffer(p.a, p.lda, t.m0, rows_a, (int64_t)t.k0 * 16, row_bytes);
    q.as = RowsBuffer(p.as, p.lda_s, t.m0, rows_a, t.k0, row_scales);
    q.b = RowsBuffer(p.b + of_b, p.ldb, w->n0, rows_b, (int64_t)t.k0 * 16, row_bytes);
    q.bs = RowsBuffer(p.bs + of_bs, p.ldb_s, w->n0, rows_b, t.k0, row_scales);
    q.va = (uint32_t)(wave * 8 + (lane >> 3)) * (uint32_t)p.lda + piece * 16;
    q.vb = (uint32_t)(wave * 8 + (lane >> 3)) * (uint32_t)p.ldb + piece * 16;
    q.vas = (uint32_t)(wave % (BM / 64) * 64 + lane) * (uint32_t)p.lda_s;
    q.vbs = (uint32_t)(wave % (BN / 64) * 64 + lane) * (uint32_t)p.ldb_s;
    q.va_last = piece_in ? q.va : kNowhere;
    q.vb_last = piece_in ? q.vb : kNowhere;
    q.step_a = (int)p.lda * 32;
    q.step_b = (int)p.ldb * 32;
    q.last = w->stages - 1;
    return true;
}

// Workgroups stay and take tile after tile: the next tile's first stage is on its way while the sums go out by way of the second
// buffer.
template <int MODE, bool F32, int BM, int BN, int PIECES>
__device__ __forceinline__ void take_tiles(const MxProductArgs& p, Walk& walk, uint8_t* lds, uint32_t done) {
    typedef TileShape<BM, BN> S;
    constexpr int FM = S::FM, FN = S::FN;
    constexpr int kStores = FM * FN * 32 * 32 * (F32 ? 4 : 2) / 1024;           // of a wave's tile in whole rows
    constexpr int kAfterStores = kStores + S::kFirstRequests < 63 ? kStores + S::kFirstRequests : 63;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 31;
    const uint32_t half = lane >> 5;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    Place at;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t at_piece = ((2 * t + half) ^ (row >> 1 & 7)) * 16;
        at.a[t] = (wm + row) * 128 + at_piece;
        at.b[t] = S::kCodesB + (wn + row) * 128 + at_piece;
    }
    at.sa = (wm + row) * 16;
    at.sb = S::kScalesB + (wn + row) * 16;
    const uint32_t lds_at = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)lds);
    const uint8_t* lds_scales = lds + S::kScalesAt;

    TileWork<S> w;
    // this workgroup's first piece, the next one that is there
    uint32_t piece = walk.first;
    auto find = [&]() {
        if (PIECES == 1) return find_work<MODE, BM, BN, 1>(p, walk, 0u, lane, wave, &w);
        for (; walk.left; piece += walk.stride, walk.left = walk.left > walk.stride ? walk.left - walk.stride : 0u) {
            walk.place(done + piece / PIECES, MODE != kMxRows, MODE == kMxDepth);
            if (find_work<MODE, BM, BN, PIECES>(p, walk, piece % PIECES, lane, wave, &w)) return true;
        }
        return false;
    };
    if (!find()) return;
    make_uniform(&w);
    request_scales<S>(lds_at + S::kScalesAt, w.q, 0, wave);
#pragma unroll
    for (int i = 0; i < S::kRequests; ++i) request_codes<S>(lds_at, w.q, 0, wave, i);
    bool stored = false;                                // kStores stores at least were issued behind the first stage's requests
    for (;;) {
#pragma unroll
        for (int i = 0; i < S::kFirstRequests; ++i) request_codes<S>(lds_at + S::kCodes, w.q, 1, wave, i);
        f32x16 acc[FM][FN];
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = f32x16{};
        Fragments<FM, FN> f0, f1;
        Scales<FM, FN> sc;
        // the first stage is here
        if (stored) __builtin_amdgcn_s_waitcnt(0x0F70 | (kAfterStores & 15) | (kAfterStores >> 4 << 14));
        else __builtin_amdgcn_s_waitcnt(0x0F70 | S::kFirstRequests);
        __syncthreads();
        read_fragments(f0, lds, at, 0);
        {
            const ScaleMask mask(w.blocks, half);
#pragma unroll
            for (int i = 0; i < FM; ++i) sc.a[i] = mask(*reinterpret_cast<const u32x2*>(lds_scales + at.sa + i * 512));
#pragma unroll
            for (int j = 0; j < FN; ++j) sc.b[j] = mask(*reinterpret_cast<const u32x2*>(lds_scales + at.sb + j * 512));
        }
        uint32_t cur = 0u;                              // buffer of the stage
        int s = 0;
        do {                                            // one stage at least
            const uint8_t *here = lds + cur, *there = lds + (S::kCodes - cur);
            // the next stage's scales: pairs of stages take turns in two buffers
            const uint8_t* sc_next = lds_scales + ((s + 1) >> 1 & 1) * S::kScales + ((s + 1) & 1) * 8;
            const uint32_t to_here = lds_at + cur, to_there = lds_at + (S::kCodes - cur);
            const ScaleMask mask(w.blocks - (s + 1) * 8, half);
            Scales<FM, FN> fresh;
            multiply_step<0, S>(acc, f0, f1, sc, fresh, here + at.a[1], here + at.b[1], sc_next + at.sa, sc_next + at.sb, to_there, w.q, s + 1, wave, mask);
            multiply_step<1, S>(acc, f1, f0, sc, fresh, here + at.a[2], here + at.b[2], sc_next + at.sa, sc_next + at.sb, to_there, w.q, s + 1, wave, mask);
            multiply_step<2, S>(acc, f0, f1, sc, fresh, here + at.a[3], here + at.b[3], sc_next + at.sa, sc_next + at.sb, to_there, w.q, s + 1, wave, mask);
            __builtin_amdgcn_s_waitcnt(0x0070);         // this wave's reads of the stage are complete, its requests of the next one too
            __syncthreads();
            if ((s & 1) == 0) request_scales<S>(lds_at + S::kScalesAt + ((s >> 1) + 1 & 1) * S::kScales, w.q, s + 2, wave);
            multiply_step<3, S>(acc, f1, f0, sc, fresh, there + at.a[0], there + at.b[0], sc_next + at.sa, sc_next + at.sb, to_here, w.q, s + 2, wave, mask);
            sc = fresh;
            cur = S::kCodes - cur;
        } while (++s < w.stages);
        // this tile's place in C, then the next tile
        const int64_t base = MODE != kMxRows ? w.t.expert * p.batch_c : 0, m0 = w.t.m0 + wm, m_end = w.t.m_end, n0 = w.n0 + wn;
        if (PIECES > 1) {
            piece += walk.stride;
            walk.left = walk.left > walk.stride ? walk.left - walk.stride : 0u;
        } else {
            walk.next(MODE != kMxRows, MODE == kMxDepth);
        }
        if (walk.left) find();
        __builtin_amdgcn_s_waitcnt(0x0070);             // the empty requests too, before the buffers are written; the last reads
        __syncthreads();
        if (walk.left) {
            make_uniform(&w);
            request_scales<S>(lds_at + S::kScalesAt, w.q, 0, wave);
#pragma unroll
            for (int i = 0; i < S::kRequests; ++i) request_codes<S>(lds_at, w.q, 0, wave, i);
        }
        settle(acc);
        stored = p.c_words;
        int own_lane = lane;                            // (as if new for every tile: its addresses are not kept in registers all along)
        asm volatile("" : "+v"(own_lane));
        store_tile<F32, FM, FN, S::kCodes / 4, MODE == kMxDepth>(p, lds + S::kCodes + wave * (S::kCodes / 4), acc, base, m0, m_end, n0, own_lane, stored);
        if (!walk.left) break;
        __syncthreads();                                // every wave has read what it put into the second buffer
    }
}

// An XCD's workgroups take its tiles round by round.  If few are left for the last round, they are cut in pieces, one for each workgroup at
// most: in quarters or halves, which take 0.3 and 0.55 times as long as a whole tile.  (16384 rows of 16 experts, 2048 x 4096, 2.25
// rounds: 90 us, 102 without; 6144 x 4096 x 8192, 1.5 rounds: 113 us, 120 without.)
template <int MODE, bool F32, int BM, int BN, int GROUPS>
__global__ __launch_bounds__(256, GROUPS) void k_mx_tile(MxProductArgs p, uint32_t total, uint32_t m_tiles, uint32_t n_tiles) {
    constexpr bool kPieces = GROUPS == 1;
    __shared__ __align__(1024) uint8_t lds[TileShape<BM, BN>::kLds];
    if (MODE == kMxRows) {                              // the host knows no more than a bound of it
        m_tiles = count_rows(p, BM);
        total = m_tiles * n_tiles;
    }
    Walk walk(total, m_tiles, n_tiles, MODE == kMxDepth);
    const uint32_t left = kPieces ? walk.mine % walk.stride : 0u, pieces = left * 4 <= walk.stride ? 4u : 2u;
    const uint32_t rest = left * 2 <= walk.stride ? left : 0u, whole = walk.mine - rest;
    if (whole > walk.first) {
        walk.left = whole - walk.first;
        walk.place(walk.first, MODE != kMxRows, MODE == kMxDepth);
        take_tiles<MODE, F32, BM, BN, 1>(p, walk, lds, 0u);
    }
    if constexpr (kPieces) {
        if (rest * pieces > walk.first) {
            __syncthreads();
            walk.left = rest * pieces - walk.first;
            if (pieces == 4) take_tiles<MODE, F32, BM / 2, BN / 2, 4>(p, walk, lds, whole);
            else take_tiles<MODE, F32, BM / 2, BN, 2>(p, walk, lds, whole);
        }
    }
}

// ---- few rows ---------------------------------------------------------------------------------------------------------
//
// Few rows of A (tokens), up to 64 per workgroup, against all of B (weights): what counts is how fast B's bytes come in.  Eight waves share a
// workgroup's 16 NT rows of B and split the depth between them, in groups of 512 (four matrix instructions); every wave has a
// group's loads on their way at once, straight into registers.  The partial sums are joined through LDS, in the order of the waves.
// (1 x 14336 x 4096: 8.0 us, 16 rows 9.9, 64 rows 14.5; B's bytes alone take 6.0 at the rate of a large copy.  The next group's loads
// ahead of the products take twice the registers and so half of the waves: 10.4 us.)
constexpr int kFewWaves = 8;
template <int MODE, int MT, int NT>
__global__ __launch_bounds__(kFewWaves * 64) void k_mx_few(MxProductArgs p, uint32_t n_tiles) {
    __shared__ __align__(16) f32x4 sums[kFewWaves][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t n_tile = blockIdx.x % n_tiles, m_tile = blockIdx.x / n_tiles;
    Tile t;
    if (!find_tile<MODE>(p, m_tile, blockIdx.z, 16 * MT, &t)) return;
    const int64_t n0 = (int64_t)n_tile * (16 * NT);
    const int64_t row_bytes = (int64_t)p.blocks * 16, row_scales = ((int64_t)p.blocks + 3) & ~3ll;
    const int64_t rows_a = min((int64_t)(16 * MT), t.m_end - t.m0), rows_b = min((int64_t)(16 * NT), p.n - n0);
    const RowsBuffer a(p.a, p.lda, t.m0, rows_a, 0, row_bytes), as(p.as, p.lda_s, t.m0, rows_a, 0, row_scales);
    const RowsBuffer b(p.b + (MODE == kMxRows ? t.expert * p.batch_b : 0), p.ldb, n0, rows_b, 0, row_bytes);
    const RowsBuffer bs(p.bs + (MODE == kMxRows ? t.expert * p.batch_bs : 0), p.ldb_s, n0, rows_b, 0, row_scales);
    const BufRsrc ra = make_buf_window(a.base, a.bytes), ras = make_buf_window(as.base, as.bytes);
    const BufRsrc rb = make_buf_window(b.base, b.bytes), rbs = make_buf_window(bs.base, bs.bytes);
    const int row = lane & 15, part = lane >> 4;
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{};
    const int groups = (p.blocks + 15) / 16;
    struct Group {
        u32x4 a[MT][4], b[NT][4], sa[MT], sb[NT];
    };
    auto load = [&](Group& v, int g) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
                v.b[j][s] = __builtin_amdgcn_raw_buffer_load_b128(rb, (uint32_t)(16 * j + row) * (uint32_t)p.ldb + part * 16 + s * 64, g * 256, 0);
            v.sb[j] = __builtin_amdgcn_raw_buffer_load_b128(rbs, (uint32_t)(16 * j + row) * (uint32_t)p.ldb_s, g * 16, 0);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
                v.a[i][s] = __builtin_amdgcn_raw_buffer_load_b128(ra, (uint32_t)(16 * i + row) * (uint32_t)p.lda + part * 16 + s * 64, g * 256, 0);
            v.sa[i] = __builtin_amdgcn_raw_buffer_load_b128(ras, (uint32_t)(16 * i + row) * (uint32_t)p.lda_s, g * 16, 0);
        }
    };
    auto multiply_group = [&](const Group& v, int g) {
        const bool ragged = g * 16 + 16 > p.blocks;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const bool in = !ragged || g * 16 + s * 4 + part < p.blocks;        // behind the last block: codes 0, scales 2^0
            uint32_t scale_b[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) scale_b[j] = in ? v.sb[j][s] >> (8 * part) : 127u;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const u32x4 codes = in ? v.a[i][s] : u32x4{0u, 0u, 0u, 0u};
                const uint32_t scale_a = in ? v.sa[i][s] >> (8 * part) : 127u;
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = mfma_mx(v.b[j][s], scale_b[j], codes, scale_a, acc[i][j]);
            }
        }
    };
    for (int g = wave; g < groups; g += kFewWaves) {
        Group now;
        load(now, g);
        multiply_group(now, g);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int f = wave; f < MT * NT; f += kFewWaves) {
        f32x4 v = sums[0][f][lane];
#pragma unroll
        for (int w = 1; w < kFewWaves; ++w) {
            const f32x4 u = sums[w][f][lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += u[e];
        }
        const int64_t m = t.m0 + f / NT * 16 + row, n = n0 + f % NT * 16 + 4 * part;
        if (m < t.m_end && n < p.n) store4(p, m * p.ldc + n, n, v);
    }
}

// Joins the parts of a split depth, in their order: four elements of a row per lane.  Bound by its launch and the caches' latency (4 us
// for eight parts of 128 x 4096).
__global__ __launch_bounds__(256) void k_mx_join(MxProductArgs p, const float* parts, int64_t ld, int64_t batch, int splits) {
    const int64_t per_row = ld / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x, m = i / per_row, n = (i - m * per_row) * 4;
    if (m >= p.m || n >= p.n) return;
    f32x4 v = *reinterpret_cast<const f32x4*>(parts + m * ld + n);
    for (int s = 1; s < splits; ++s) {
        const f32x4 u = *reinterpret_cast<const f32x4*>(parts + s * batch + m * ld + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += u[e];
    }
    store4(p, m * p.ldc + n, n, v);
}

}  // namespace

// Which kernel a product of a given size takes.  Times in us, measured on whole and partly filled cards: a stage of a 256 x 256 tile
// 1.9, of half of one 1.05, of two 128 x 128 tiles on a CU 1.29, of one 0.56, and what a tile costs besides 8, 6 and 5.  (In large
// tiles and in small ones, us: 4096 x 4096 x 4096 38 and 47, 4096 x 5120 x 512 16.8 and 17.4, 2048 x 4096 x 4096 30.1 and 27.6,
// 1024 x 4096 x 4096 27.9 and 17.1.)
struct ProductPlan {
    enum { kFew, kSmallTiles, kLargeTiles } kind;
    int splits;                         // parts of the depth
    int mt, nt;                         // kFew: 16 rows of A and of B of a workgroup
};
// The more rows of B a workgroup takes, the less often A's are read (64 x 14336 x 4096: 30.5 us with 16, 18.6 with 32, 14.5 with 64), but
// the CUs want 160 workgroups at least (64 x 4096 x 4096: 8.6, 10.0, 13.4).  `rows`: of B, times the workgroups for A's.
static int few_nt(double rows) { return rows < 160 * 32 ? 1 : rows < 160 * 64 ? 2 : 4; }

// Tiles of `height` rows: of a product, of all experts' results, or to expect in the segments of experts, if the choices fall on them at
// random: the mean of what a standard deviation less and one more choices for each would make.
static double tile_rows(int mode, const MxProductArgs& p, int height) {
    if (mode != kMxRows) return (double)((p.m + height - 1) / height) * (mode == kMxDepth ? p.n_experts : 1);
    const double used = std::max(std::min(p.n_experts, p.choices), 1), each = std::max((double)p.choices / used, 1.0);
    double sum = 0;
    for (const double rows : {std::max(each - std::sqrt(each), 1.0), each + std::sqrt(each)})
        sum += std::ceil(std::ceil(rows / p.align) * p.align / height);
    return used * sum / 2;
}

static ProductPlan plan_product(int mode, const MxProductArgs& p) {
    const int64_t m = p.m, n = p.n, blocks = p.blocks;
    // (More than 32 rows and a long depth for few workgroups: parts of the depth are better.  64 x 4096 x 14336: 22.5 us, 18.8 in tiles;
    // 64 x 4096 x 8192: 15.3 and 17.3.)  Up to four rows are read often at little cost, so that more
    // workgroups are worth it (with 16 rows of B and by few_nt, 1, 2 and 4 rows, n from 5200 to 20000, k from 512 to 8192: up to 20 %
    // less, 1 x 20000 x 8192 21.8 and 26.2 us, 1 x 8192 x 4096 5.8 and 6.2, 4 x 14336 x 512 3.8 and 4.6; at the worst 8 % more,
    // 4 x 14336 x 4096 9.4 and 8.5 to 9.3, 4 x 5200 x 8192 9.7 and 9.0).
    if (mode == kMxDense && m <= 64 && !(m > 32 && n < 160 * 32 && blocks > 320))
        return {ProductPlan::kFew, 1, m <= 16 ? 1 : m <= 32 ? 2 : 4, m <= 4 && n < 160 * 128 ? 1 : few_nt((double)n)};
    // Rows of experts: every expert's matrix is read once in tiles, once for each 16 of its rows otherwise.  (Experts of 2048 x 4096, us
    // for few rows and in tiles: 64 experts with 2 rows each 48.5 and 55, with 4 60.6 and 59.8, with 16 90 and 62; 8 experts of
    // 4096 x 4096, too few tiles for the CUs, with 12 rows each 21.4 and 22.2, with 16 24.5 and 22.3.)
    if (mode == kMxRows && m <= (std::min<int64_t>(m, p.n_experts) * ((n + 127) / 128) <= 512 ? 12 : 4) * p.n_experts)
        return {ProductPlan::kFew, 1, 1, std::min<int64_t>(m, p.n_experts) * n < 160 * 32 ? 1 : 2};
    // Workgroups of 64 rows, if there are no more of them than CUs and the depth is not long (for few rows and in tiles, us of GPU time:
    // 100 x 2700 x 2700 7.1 and 13.6, 128 x 4096 x 4096 10.4 and 16.0, 512 x 2048 x 2048 8.4 and 8.9; with 448 workgroups 128 x 14336 x
    // 4096 24.5 and 20.8; with a depth of 8192 128 x 1024 x 8192 14.1 and 13.2).
    if (mode != kMxDepth && blocks < 256) {
        const double rows = tile_rows(mode, p, 64);
        const int nt = few_nt(rows * n);
        if (rows * (double)((n + 16 * nt - 1) / (16 * nt)) <= 256) return {ProductPlan::kFew, 1, 4, nt};
    }
    const double stages = std::ceil((double)blocks / 8 / (mode == kMxDepth ? std::max(p.n_experts, 1) : 1));
    const double large = std::ceil(tile_rows(mode, p, 256) * (double)((n + 255) / 256)), small = std::ceil(tile_rows(mode, p, 128) * (double)((n + 127) / 128));
    const double rest = std::fmod(small, 512), left = std::fmod(large, 256);
    const double in_large = std::floor(large / 256) * (1.9 * stages + 8) +
                            (left == 0 ? 0.0 : left > 128 || large < 256 ? 1.9 * stages + 8 : left > 64 ? 1.05 * stages + 6 : 0.56 * stages + 5);
    const double in_small = std::floor(small / 512) * (1.29 * stages + 5) + (rest == 0 ? 0.0 : (rest <= 256 ? 0.56 : 1.29) * stages + 5);
    if (in_large <= in_small) return {ProductPlan::kLargeTiles, 1, 0, 0};
    // Few tiles and a long depth: parts of it on idle CUs.  They are written and read again at about 4 TB/s, and joining them is a
    // launch of its own (128 x 4096 x 14336: 18.5 us in eight parts, 42 in one; 512 x 4096 x 4096: 18.2 in two, 13.9 in one).
    ProductPlan best{ProductPlan::kSmallTiles, 1, 0, 0};
    double least = in_small;
    if (mode == kMxDense && small <= 128)
        for (int splits = 2; splits * small <= 256 && splits <= 32; splits *= 2) {
            const double time = std::ceil(stages / splits) * 0.56 + 9 + (double)splits * (double)m * (double)n * 8e-6 / 4;
            if (time < least) { least = time; best.splits = splits; }
        }
    // Parts of whole stages: no more of them than get any (100 x 257 x 8200: 33 stages in 11 parts of three, not in 16).  The first block
    // of each is then a multiple of 8, so that its scales begin at a whole word.
    if (best.splits > 1) {
        const int all = (int)((blocks + 7) / 8), each = (all + best.splits - 1) / best.splits;
        best.splits = (all + each - 1) / each;
    }
    return best;
}
static int64_t part_ld(int64_t n) { return (n + 3) / 4 * 4; }

size_t mx_product_workspace(int64_t m, int64_t n, int32_t blocks) {
    MxProductArgs p{};
    p.m = m; p.n = n;
    p.blocks = blocks;
    const int splits = plan_product(kMxDense, p).splits;
    return splits == 1 ? 0 : (size_t)splits * m * part_ld(n) * 4;
}

constexpr int64_t kCus = 256;            // of an MI355X
template <bool F32, int BM, int BN, int GROUPS>
static hipError_t launch_tiles(int mode, const MxProductArgs& p, hipStream_t st) {
    const int64_t n_tiles = (p.n + BN - 1) / BN;
    int64_t m_tiles = (p.m + BM - 1) / BM;
    if (mode == kMxRows) m_tiles = p.m / BM + std::min<int64_t>(p.n_experts, p.m);
    const int64_t total = n_tiles * m_tiles * (mode == kMxDepth ? p.n_experts : p.splits);
    if (total > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)std::min<int64_t>(total, kCus * GROUPS));
    const uint32_t tiles = (uint32_t)total, mt = (uint32_t)m_tiles, nt = (uint32_t)n_tiles;
    if (mode == kMxDense) k_mx_tile<kMxDense, F32, BM, BN, GROUPS><<<grid, dim3(256), 0, st>>>(p, tiles, mt, nt);
    else if (mode == kMxRows) k_mx_tile<kMxRows, F32, BM, BN, GROUPS><<<grid, dim3(256), 0, st>>>(p, tiles, mt, nt);
    else k_mx_tile<kMxDepth, F32, BM, BN, GROUPS><<<grid, dim3(256), 0, st>>>(p, tiles, mt, nt);
    return hipGetLastError();
}

template <int MT, int NT>
static hipError_t launch_few(int mode, const MxProductArgs& p, hipStream_t st) {
    const int64_t n_tiles = (p.n + 16 * NT - 1) / (16 * NT);
    int64_t m_tiles = (p.m + 16 * MT - 1) / (16 * MT);
    if (mode == kMxRows) m_tiles = p.m / (16 * MT) + std::min<int64_t>(p.n_experts, p.m);
    if (n_tiles * m_tiles > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)(n_tiles * m_tiles)), block(kFewWaves * 64);
    if (mode == kMxDense) k_mx_few<kMxDense, MT, NT><<<grid, block, 0, st>>>(p, (uint32_t)n_tiles);
    else if constexpr (MT == 4 || (MT == 1 && NT <= 2)) k_mx_few<kMxRows, MT, NT><<<grid, block, 0, st>>>(p, (uint32_t)n_tiles);
    else return hipErrorInvalidValue;                   // no kernel of this shape: plan_product asks for none
    return hipGetLastError();
}

static bool near_rows(const MxProductArgs& p) {         // 256 rows of either operand within 32-bit offsets
    return 256 * std::max(std::max(p.lda, p.ldb), std::max(p.lda_s, p.ldb_s)) < 0x7FFFFFFFll;
}
static hipError_t launch_all_tiles(int mode, MxProductArgs p, bool large, hipStream_t st) {
    const int64_t size = p.f32 ? 4 : 2;
    p.c_words = ((reinterpret_cast<uintptr_t>(p.c) | (uintptr_t)(p.ldc * size) | (uintptr_t)(p.batch_c * size)) & 3) == 0 && 256 * p.ldc * size < 0x7FFFFFFFll;
    p.c_lines = ((reinterpret_cast<uintptr_t>(p.c) | (uintptr_t)(p.ldc * size) | (uintptr_t)(p.batch_c * size)) & 127) == 0;
    if (large) return p.f32 ? launch_tiles<true, 256, 256, 1>(mode, p, st) : launch_tiles<false, 256, 256, 1>(mode, p, st);
    return p.f32 ? launch_tiles<true, 128, 128, 2>(mode, p, st) : launch_tiles<false, 128, 128, 2>(mode, p, st);
}

hipError_t launch_mx_product(int mode, MxProductArgs p, void* workspace, hipStream_t st) {
    p.splits = 1;
    if (near_rows(p)) {
        const ProductPlan plan = plan_product(mode, p);
        if (plan.kind == ProductPlan::kFew) {
            if (plan.mt == 1) return plan.nt == 1 ? launch_few<1, 1>(mode, p, st) : plan.nt == 2 ? launch_few<1, 2>(mode, p, st) : launch_few<1, 4>(mode, p, st);
            if (plan.mt == 2) return plan.nt == 1 ? launch_few<2, 1>(mode, p, st) : plan.nt == 2 ? launch_few<2, 2>(mode, p, st) : launch_few<2, 4>(mode, p, st);
            return plan.nt == 1 ? launch_few<4, 1>(mode, p, st) : plan.nt == 2 ? launch_few<4, 2>(mode, p, st) : launch_few<4, 4>(mode, p, st);
        }
        if (plan.splits == 1) return launch_all_tiles(mode, p, plan.kind == ProductPlan::kLargeTiles, st);
        MxProductArgs part = p;
        part.c = workspace;
        part.ldc = part_ld(p.n);
        part.batch_c = p.m * part.ldc;
        part.f32 = 1;
        part.splits = plan.splits;
        const hipError_t e = launch_all_tiles(mode, part, false, st);
        if (e != hipSuccess) return e;
        const int64_t lanes = p.m * (part.ldc / 4);
        const dim3 grid((uint32_t)((lanes + 255) / 256));
        k_mx_join<<<grid, dim3(256), 0, st>>>(p, static_cast<const float*>(workspace), part.ldc, part.batch_c, plan.splits);
        return hipGetLastError();
    }
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
