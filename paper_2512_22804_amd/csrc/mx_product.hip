// Products of microscaled 4-bit operands on the matrix cores.
#include <algorithm>

#include "mx_device.h"
#include "mx_launch.h"

namespace mor {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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
// A workgroup of four waves forms BM x BN elements of C, each wave a quarter.  A stage is 128 of the depth, one matrix
// instruction deep: 64 bytes of codes and 4 of scales per row, loaded from global memory straight into one of four LDS buffers.
// While stage s is multiplied, its later fragments and the first ones of stage s + 1 are read from LDS into registers, stage
// s + 2 is on its way and stage s + 3 is requested into the buffer that stage s - 1 left; one barrier per stage.
//
// The four 16-byte pieces of a row lie permuted: piece j of row r at j ^ (r / 2 % 4), so that eight rows' pieces of the same
// depth, which one LDS cycle serves, fall into different banks.  Rows beyond the operand's last lie outside the buffer
// resource's range and arrive as zeros; so do the pieces behind a row's last block, whose lanes request an address out of range
// in the last stage, and stages beyond the last, whose range is empty.  The scale bytes behind the last block, loaded four at
// a time, are replaced by 2^0: whatever they hold, a NaN too, counts for nothing.

typedef __attribute__((address_space(3))) void lds_void;

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
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(int step, bool exists) const {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base) + step, 0, exists ? max(bytes - step, 0) : 0, 0x00020000);
    }
};

template <int BM, int BN>
struct TileShape {
    static constexpr int FM = BM / 32, FN = BN / 32;    // fragments of 16 rows of a wave
    static constexpr int kCodesB = BM * 64, kScalesA = (BM + BN) * 64, kScalesB = kScalesA + BM * 4, kBytes = kScalesB + BN * 4;
    static constexpr int kRequests = (BM + BN) / 64 + (BM + BN) / 256;      // of one wave and stage
};

// What a lane adds to the stage's base to request its pieces.
struct Request {
    RowsBuffer a, as, b, bs;
    uint32_t va, vb, vas, vbs;          // offset in the first group of rows
    uint32_t va_last, vb_last;          // the same in the last stage
    int step_a, step_b, step_as, step_bs;       // bytes between the groups of a wave
    int last;
};

// Wave w loads the codes of rows 16 (w + 4 i) .. + 15 and the scales of rows 64 (w + 4 i) .. + 63.
template <int BM, int BN>
__device__ __forceinline__ void request_stage(uint8_t* lds, const Request& q, int stage, int wave) {
    typedef TileShape<BM, BN> S;
    const bool exists = stage <= q.last;
    const __amdgpu_buffer_rsrc_t ra = q.a.at(stage * 64, exists), rb = q.b.at(stage * 64, exists);
    const __amdgpu_buffer_rsrc_t ras = q.as.at(stage * 4, exists), rbs = q.bs.at(stage * 4, exists);
    const uint32_t va = stage == q.last ? q.va_last : q.va, vb = stage == q.last ? q.vb_last : q.vb;
#pragma unroll
    for (int i = 0; i < BM / 64; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(lds + (wave + 4 * i) * 1024), 16, va, i * q.step_a, 0, 0);
#pragma unroll
    for (int i = 0; i < BN / 64; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_void*)(lds + S::kCodesB + (wave + 4 * i) * 1024), 16, vb, i * q.step_b, 0, 0);
    if (BM >= 256) __builtin_amdgcn_raw_ptr_buffer_load_lds(ras, (lds_void*)(lds + S::kScalesA + wave * 256), 4, q.vas, 0, 0, 0);
    if (BN >= 256) __builtin_amdgcn_raw_ptr_buffer_load_lds(rbs, (lds_void*)(lds + S::kScalesB + wave * 256), 4, q.vbs, 0, 0, 0);
    if (BM == 128 && BN == 128) {       // two waves the scales of A, two those of B, which follow them in LDS
        if (wave < 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(ras, (lds_void*)(lds + S::kScalesA + wave * 256), 4, q.vas, 0, 0, 0);
        else __builtin_amdgcn_raw_ptr_buffer_load_lds(rbs, (lds_void*)(lds + S::kScalesA + wave * 256), 4, q.vbs, 0, 0, 0);
    }
}

// A lane's places in a buffer.
struct Place {
    uint32_t a, b, sa, sb;
};

template <int FM, int FN>
struct Fragments {
    u32x4 a0, a1, b[FN];                // the first two of A
    uint32_t sa[FM], sb[FN];
};
template <int BM, int BN>
__device__ __forceinline__ void read_first(Fragments<BM / 32, BN / 32>& f, const uint8_t* lds, const Place& at) {
#pragma unroll
    for (int j = 0; j < BN / 32; ++j) { f.b[j] = *reinterpret_cast<const u32x4*>(lds + at.b + j * 1024); f.sb[j] = lds[at.sb + j * 64]; }
    f.a0 = *reinterpret_cast<const u32x4*>(lds + at.a);
    f.a1 = *reinterpret_cast<const u32x4*>(lds + at.a + 1024);
#pragma unroll
    for (int i = 0; i < BM / 32; ++i) f.sa[i] = lds[at.sa + i * 64];
}

// Four matrix instructions.  The compiler keeps the accumulators of a 128 x 128 wave in place only if told to: with the builtin it
// gives sums and addends different registers, which do not suffice (256 of 512 are accumulators), and moves them about.  As it
// does not look into the text, the two wait states between a vector instruction that writes an operand and a matrix instruction
// that reads it stand there, and settle() below stands before the first other use of the sums.
#define MOR_MFMA(C, B, SB) "v_mfma_scale_f32_16x16x128_f8f6f4 " C ", " B ", %8, " C ", " SB ", %13 op_sel_hi:[0,0,0] cbsz:4 blgp:4\n\t"
__device__ __forceinline__ void mfma4(f32x4& c0, f32x4& c1, f32x4& c2, f32x4& c3, u32x4 a, uint32_t sa, u32x4 b0, u32x4 b1, u32x4 b2, u32x4 b3,
                                      uint32_t sb0, uint32_t sb1, uint32_t sb2, uint32_t sb3) {
    asm("s_nop 1\n\t" MOR_MFMA("%0", "%4", "%9") MOR_MFMA("%1", "%5", "%10") MOR_MFMA("%2", "%6", "%11") MOR_MFMA("%3", "%7", "%12")
        : "+a"(c0), "+a"(c1), "+a"(c2), "+a"(c3)
        : "v"(b0), "v"(b1), "v"(b2), "v"(b3), "v"(a), "v"(sb0), "v"(sb1), "v"(sb2), "v"(sb3), "v"(sa));
}
#undef MOR_MFMA
// The last matrix instructions (four passes of four cycles) have written their sums.
__device__ __forceinline__ void settle(f32x4& c0, f32x4& c1, f32x4& c2, f32x4& c3) {
    asm volatile("s_nop 15\n\ts_nop 15" : "+a"(c0), "+a"(c1), "+a"(c2), "+a"(c3));
}

// One stage: `cur` holds its first fragments; `next` receives those of the stage in `lds_next`.
template <int BM, int BN>
__device__ __forceinline__ void multiply_stage(f32x4 (&acc)[BM / 32][BN / 32], Fragments<BM / 32, BN / 32>& cur, Fragments<BM / 32, BN / 32>& next,
                                               const uint8_t* lds, const uint8_t* lds_next, uint8_t* lds_free, const Place& at, const Request& q,
                                               int stage, int wave, bool keep_last) {
    constexpr int FM = BM / 32, FN = BN / 32, kRequests = TileShape<BM, BN>::kRequests;
    static_assert(FM == FN, "one fragment of each operand is read per step");
    __builtin_amdgcn_s_waitcnt(0x0F70 | kRequests);     // all but the latest stage's requests have arrived
    __syncthreads();
    request_stage<BM, BN>(lds_free, q, stage + 3, wave);
    const bool keep = stage + 1 < q.last || keep_last;
    u32x4 a0 = cur.a0, a1 = cur.a1;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const u32x4 a = a0;
        a0 = a1;
        a1 = *reinterpret_cast<const u32x4*>(i + 2 < FM ? lds + at.a + (i + 2) * 1024 : lds_next + at.a + (i + 2 - FM) * 1024);
        next.b[i] = *reinterpret_cast<const u32x4*>(lds_next + at.b + i * 1024);
        const uint32_t sb = lds_next[at.sb + i * 64], sa = lds_next[at.sa + i * 64];
        next.sb[i] = keep ? sb : 127u;
        next.sa[i] = keep ? sa : 127u;
#pragma unroll
        for (int j = 0; j < FN; j += 4)
            mfma4(acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3], a, cur.sa[i], cur.b[j], cur.b[j + 1], cur.b[j + 2], cur.b[j + 3],
                  cur.sb[j], cur.sb[j + 1], cur.sb[j + 2], cur.sb[j + 3]);
        __builtin_amdgcn_sched_barrier(0);      // the reads stay spread over the matrix instructions
    }
    next.a0 = a0;
    next.a1 = a1;
}

template <int MODE, int BM, int BN>
__global__ __launch_bounds__(256, 1) void k_mx_tile(MxProductArgs p, uint32_t m_tiles, uint32_t n_tiles) {
    typedef TileShape<BM, BN> S;
    constexpr int FM = S::FM, FN = S::FN;
    __shared__ __align__(1024) uint8_t buf0[S::kBytes];
    __shared__ __align__(1024) uint8_t buf1[S::kBytes];
    __shared__ __align__(1024) uint8_t buf2[S::kBytes];
    __shared__ __align__(1024) uint8_t buf3[S::kBytes];
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
              (int)p.lda * 64, (int)p.ldb * 64, (int)p.lda_s * 256, (int)p.ldb_s * 256, stages - 1};
    q.va_last = piece_in ? q.va : kNowhere;
    q.vb_last = piece_in ? q.vb : kNowhere;

    const int row = lane & 15, part = lane >> 4;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    const uint32_t at_piece = (part ^ (row >> 1 & 3)) * 16;
    const Place at{(uint32_t)(wm + row) * 64 + at_piece, (uint32_t)S::kCodesB + (wn + row) * 64 + at_piece,
                   (uint32_t)S::kScalesA + (wm + row) * 4 + part, (uint32_t)S::kScalesB + (wn + row) * 4 + part};
    const bool keep_last = (stages - 1) * 4 + part < blocks;

    f32x4 acc[FM][FN] = {};
    if (stages > 0) {
        Fragments<FM, FN> f0, f1;
        request_stage<BM, BN>(buf0, q, 0, wave);
        request_stage<BM, BN>(buf1, q, 1, wave);
        request_stage<BM, BN>(buf2, q, 2, wave);
        __builtin_amdgcn_s_waitcnt(0x0F70 | (2 * S::kRequests & 15) | (2 * S::kRequests >> 4 << 14));
        __syncthreads();
        read_first<BM, BN>(f0, buf0, at);
        if (stages == 1 && !keep_last) {
#pragma unroll
            for (int i = 0; i < FM; ++i) f0.sa[i] = 127u;
#pragma unroll
            for (int j = 0; j < FN; ++j) f0.sb[j] = 127u;
        }
        // (One way out of the loop: with more the compiler moves accumulators between registers.)
        for (int s = 0; s < stages; s += 4) {
            multiply_stage<BM, BN>(acc, f0, f1, buf0, buf1, buf3, at, q, s, wave, keep_last);
            if (s + 1 < stages) multiply_stage<BM, BN>(acc, f1, f0, buf1, buf2, buf0, at, q, s + 1, wave, keep_last);
            if (s + 2 < stages) multiply_stage<BM, BN>(acc, f0, f1, buf2, buf3, buf1, at, q, s + 2, wave, keep_last);
            if (s + 3 < stages) multiply_stage<BM, BN>(acc, f1, f0, buf3, buf0, buf2, at, q, s + 3, wave, keep_last);
        }
        __builtin_amdgcn_s_waitcnt(0x0F70);             // the empty requests too, before the LDS is another workgroup's
    }
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; j += 4) settle(acc[i][j], acc[i][j + 1], acc[i][j + 2], acc[i][j + 3]);

#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t m = t.m0 + wm + 16 * i + row;
        if (m >= t.m_end) continue;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t n = n0 + wn + 16 * j + 4 * part;
            if (n < p.n) store4(p, (MODE == kMxDepth ? t.expert * p.batch_c : 0) + m * p.ldc + n, n, acc[i][j]);
        }
    }
}

}  // namespace

size_t mx_product_workspace(int64_t, int64_t, int64_t) { return 0; }

template <int BM, int BN>
static hipError_t launch_tiles(int mode, const MxProductArgs& p, hipStream_t st) {
    const int64_t n_tiles = (p.n + BN - 1) / BN;
    int64_t m_tiles = (p.m + BM - 1) / BM;
    if (mode == kMxRows) m_tiles = p.m / BM + std::min<int64_t>(p.n_experts, p.m);
    const int64_t total = n_tiles * m_tiles * (mode == kMxDepth ? p.n_experts : 1);
    if (total > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)total);
    if (mode == kMxDense) k_mx_tile<kMxDense, BM, BN><<<grid, dim3(256), 0, st>>>(p, (uint32_t)m_tiles, (uint32_t)n_tiles);
    else if (mode == kMxRows) k_mx_tile<kMxRows, BM, BN><<<grid, dim3(256), 0, st>>>(p, (uint32_t)m_tiles, (uint32_t)n_tiles);
    else k_mx_tile<kMxDepth, BM, BN><<<grid, dim3(256), 0, st>>>(p, (uint32_t)m_tiles, (uint32_t)n_tiles);
    return hipGetLastError();
}

hipError_t launch_mx_product(int mode, const MxProductArgs& p, void*, hipStream_t st) {
    // a tile's rows are addressed with 32-bit offsets
    const bool near = 256 * std::max(std::max(p.lda, p.ldb), std::max(p.lda_s, p.ldb_s)) < 0x7FFFFFFFll;
    if (near && p.m > 128) return launch_tiles<256, 256>(mode, p, st);
    if (near && p.m > 32) return launch_tiles<128, 128>(mode, p, st);
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
