// Tokens sorted by expert and back: the order, rows gathered into it, weighted sums out of it, and the gradients.
#include <algorithm>

#include "mx_device.h"
#include "mx_launch.h"

namespace mor {
namespace {

constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64;
constexpr int kMaxExperts = 1024;       // one lane each
constexpr int64_t kSortLone = 2048;     // choices that one workgroup sorts alone: 5.2 us for 1332, 9.6 for 4000; two launches 7.7
constexpr int64_t kSortChunks = 256;    // workgroups at most, each of which sums up the counts of all

__device__ __forceinline__ uint32_t expert_of(const int32_t* ids, int64_t i, int64_t n, uint32_t experts) {
    const uint32_t e = i < n ? (uint32_t)ids[i] : experts;
    return e < experts ? e : experts;   // dropped
}

// Choices of each expert in each chunk; integer sums, so their order does not matter.
__global__ __launch_bounds__(kSortThreads) void k_expert_count(const int32_t* ids, int64_t choices, uint32_t experts, uint32_t* counts, int rounds) {
    __shared__ uint32_t hist[kMaxExperts + 1];
    for (uint32_t e = threadIdx.x; e <= experts; e += kSortThreads) hist[e] = 0u;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * rounds * kSortThreads;
    for (int j = 0; j < rounds; ++j) {
        const uint32_t e = expert_of(ids, i0 + j * kSortThreads + threadIdx.x, choices, experts);
        if (e < experts) atomicAdd(&hist[e], 1u);
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < experts; e += kSortThreads) counts[(int64_t)blockIdx.x * experts + e] = hist[e];
}

// Sum over the 1024 lanes before this one (an exclusive scan); `wave_sums` [kSortWaves].
__device__ __forceinline__ uint32_t scan_before(uint32_t v, uint32_t* wave_sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t upto = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t other = (uint32_t)__shfl_up((int)upto, d);
        if (lane >= d) upto += other;
    }
    if (lane == 63) wave_sums[wave] = upto;
    __syncthreads();
    uint32_t before = 0u;
    for (int w = 0; w < wave; ++w) before += wave_sums[w];
    return before + upto - v;
}

// The places of a chunk's choices.  LONE: one chunk in all, which is counted here; else the counts of every chunk are read.
// Lane e holds expert e's sums.  Within 64 choices the lanes of one expert find each other by ballots over the bits of its number,
// so a choice's rank needs no atomic and the order is the choices' own.  Bound by latency: loads that depend on each other, a scan
// and a few barriers (8192 tokens, 2 of 16 experts: 8.0 us with the count, 32768 tokens, 8 of 64: 11.8 us).
template <bool LONE>
__global__ __launch_bounds__(kSortThreads) void k_expert_place(const int32_t* ids, int64_t choices, const uint32_t* counts, MxOrder o, int rounds) {
    __shared__ uint32_t next[kMaxExperts + 1];              // slot of the expert's next choice
    __shared__ uint32_t wave_sums[kSortWaves];
    __shared__ uint8_t in_wave[kSortWaves][kMaxExperts];    // choices of the expert among a wave's 64
    const uint32_t experts = (uint32_t)o.n_experts, e = threadIdx.x, chunks = gridDim.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t i0 = (int64_t)blockIdx.x * rounds * kSortThreads;
    uint32_t id = expert_of(ids, i0 + threadIdx.x, choices, experts);       // the first round's, on its way as early as can be
    uint32_t total = 0u, earlier = 0u;
    if (LONE) {
        if (e <= experts) next[e] = 0u;
        if (e == 0) next[experts] = 0u;
        __syncthreads();
        for (int64_t i = threadIdx.x; i < choices; i += kSortThreads) {
            const uint32_t id = expert_of(ids, i, choices, experts);
            if (id < experts) atomicAdd(&next[id], 1u);
        }
        __syncthreads();
        if (e < experts) total = next[e];
        __syncthreads();
    } else {
        // the counts of all chunks, as many lanes to an expert as there are
        __shared__ uint32_t sums[2][kMaxExperts];
        if (e < experts) sums[0][e] = sums[1][e] = 0u;
        __syncthreads();
        const uint32_t each = kSortThreads / experts;           // chunks at a time
        if (e < each * experts) {
            const uint32_t of = e % experts;
            uint32_t all = 0u, before = 0u;
            for (uint32_t c = e / experts; c < chunks; c += each) {
                const uint32_t n = counts[(int64_t)c * experts + of];
                if (c < blockIdx.x) before += n;
                all += n;
            }
            if (all) atomicAdd(&sums[0][of], all);
            if (before) atomicAdd(&sums[1][of], before);
        }
        __syncthreads();
        if (e < experts) { total = sums[0][e]; earlier = sums[1][e]; }
    }
    const uint32_t padded = (total + o.align - 1) / o.align * o.align;
    const uint32_t start = scan_before(padded, wave_sums);
    if (e < experts) next[e] = start + earlier;
    if (blockIdx.x == 0) {
        if (e < experts) o.offsets[e] = (int32_t)start;
        if (e == experts - 1) o.offsets[experts] = (int32_t)(start + padded);
    }
    // empty slots: a wave for those of an expert, those behind the last one shared out over all workgroups
    __shared__ uint32_t empty[kMaxExperts][2];
    if (e < experts) { empty[e][0] = start + total; empty[e][1] = start + padded; }
    __shared__ uint32_t end;
    if (e == experts - 1) end = start + padded;
    __syncthreads();
    if (o.align > 1)
        for (uint32_t x = blockIdx.x * kSortWaves + wave; x < experts; x += chunks * kSortWaves)
            for (uint32_t s = empty[x][0] + lane; s < empty[x][1]; s += 64)
                if (s < (uint32_t)o.capacity) o.src[s] = -1;
    for (int64_t s = (int64_t)end + blockIdx.x * kSortThreads + threadIdx.x; s < o.capacity; s += (int64_t)chunks * kSortThreads) o.src[s] = -1;

    for (int j = 0; j < rounds; ++j) {
        const int64_t i = i0 + j * kSortThreads + threadIdx.x;
        if (i0 + j * kSortThreads >= choices) break;
        for (uint32_t q = lane; q < (experts + 3) / 4; q += 64) reinterpret_cast<uint32_t*>(in_wave[wave])[q] = 0u;
        if (j > 0) id = expert_of(ids, i, choices, experts);
        uint64_t same = __ballot(id < experts);
        for (uint32_t bit = 1u; bit < experts; bit <<= 1) {
            const uint64_t set = __ballot((id & bit) != 0u);
            same &= (id & bit) ? set : ~set;
        }
        const uint32_t rank = __popcll(same & ((1ull << lane) - 1ull));
        if (id < experts && rank == 0) in_wave[wave][id] = (uint8_t)__popcll(same);
        __syncthreads();
        if (id < experts) {
            uint32_t slot = next[id] + rank;
            for (int w = 0; w < wave; ++w) slot += in_wave[w][id];
            o.slot_of[i] = (int32_t)slot;
            if (slot < (uint32_t)o.capacity) o.src[slot] = (int32_t)i;
        } else if (i < choices) o.slot_of[i] = -1;
        if (j + 1 == rounds) break;
        __syncthreads();
        if (e < experts) {
            uint32_t n = 0u;
            for (int w = 0; w < kSortWaves; ++w) n += in_wave[w][e];
            next[e] += n;
        }
        __syncthreads();
    }
}

__device__ __forceinline__ u32x4 narrow8(const float (&f)[8]) {
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = bf16_of(f[2 * j]) | (bf16_of(f[2 * j + 1]) << 16);
    return v;
}

// Elements of a row that one wave moves: two chunks per lane.  The spans of a row follow each other, not the rows of a span (sums of two
// rows of 4096 for each of 8192 tokens: 33 us, 42 the other way).
constexpr int kRowSpan = 1024;

// One wave per slot and span.  Bound by the bytes written (8192 tokens of 4096 into 18432 slots: 39 us, 5.6 TB/s of what is read
// and written once).
template <bool STREAM>
__global__ __launch_bounds__(256) void k_expert_gather(const uint16_t* x, int64_t ld_x, int64_t d, MxOrder o, uint16_t* xs, int64_t ld_xs, uint32_t spans) {
    const uint32_t group = blockIdx.x / spans, span = blockIdx.x - group * spans;
    const int64_t slot = (int64_t)group * 4 + (threadIdx.x >> 6);
    if (slot >= o.capacity) return;
    const uint32_t choice = (uint32_t)o.src[slot], choices = (uint32_t)o.tokens * (uint32_t)o.top_k;
    const uint16_t* row = choice < choices ? x + (int64_t)(choice / (uint32_t)o.top_k) * ld_x : nullptr;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t c = (int64_t)span * kRowSpan + h * 512 + (threadIdx.x & 63) * 8;
        if (c < d) store8<STREAM>(xs + slot * ld_xs, c, d, row ? load8(row, c, d) : u32x4{0u, 0u, 0u, 0u});
    }
}

// Eight elements of a row from column c on as they are in memory, BF16 or binary32, and their values.  Loading and using are apart, so
// that several rows can be on their way.
template <class T, bool STREAM>
struct Piece;
template <bool STREAM>
struct Piece<uint16_t, STREAM> {
    u32x4 raw;
    __device__ __forceinline__ void load(const uint16_t* row, int64_t c, int64_t d) { raw = load8_start<STREAM>(row, c, d); }
    __device__ __forceinline__ void clear() { raw = u32x4{0u, 0u, 0u, 0u}; }
    __device__ __forceinline__ void values(int64_t c, int64_t d, float (&f)[8]) const { widen8(c < d ? load8_end(raw, c, d) : raw, f); }
};
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_anywhere __attribute__((aligned(4)));
template <bool STREAM>
struct Piece<float, STREAM> {
    f32x4 raw[2];
    __device__ __forceinline__ void load(const float* row, int64_t c, int64_t d) {
        const f32x4_anywhere* p = reinterpret_cast<const f32x4_anywhere*>(row + c);
        if (c + 8 <= d) {
            raw[0] = STREAM ? __builtin_nontemporal_load(p) : p[0];
            raw[1] = STREAM ? __builtin_nontemporal_load(p + 1) : p[1];
            return;
        }
        clear();
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < d) raw[j / 4][j % 4] = row[c + j];
    }
    __device__ __forceinline__ void clear() { raw[0] = raw[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }
    __device__ __forceinline__ void values(int64_t, int64_t, float (&f)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = raw[j / 4][j % 4];
    }
};
template <bool STREAM>
__device__ __forceinline__ void store_values(uint16_t* row, int64_t c, int64_t d, const float (&f)[8]) { store8<STREAM>(row, c, d, narrow8(f)); }
template <bool STREAM>
__device__ __forceinline__ void store_values(float* row, int64_t c, int64_t d, const float (&f)[8]) {
    f32x4_anywhere* p = reinterpret_cast<f32x4_anywhere*>(row + c);
    const f32x4 low = {f[0], f[1], f[2], f[3]}, high = {f[4], f[5], f[6], f[7]};
    if (c + 8 <= d) {
        if (STREAM) { __builtin_nontemporal_store(low, p); __builtin_nontemporal_store(high, p + 1); }
        else { p[0] = low; p[1] = high; }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (c + j < d) row[c + j] = f[j];
}

// One wave per token and span: a sum over the token's choices in binary32, in their order, so no atomics.  Bound by the rows read (two of
// 4096 for each of 8192 tokens: 33 us, 6.1 TB/s).  Rows are BF16 or binary32, as a product writes them: BF16 is a rounding more (2^-9 of
// each row's elements, where their 4-bit factors carry 2^-3) for half of the bytes that product and sum move.
template <class IN, class OUT, bool WEIGHTS, bool STREAM>
__global__ __launch_bounds__(256) void k_expert_combine(const IN* ys, int64_t ld_ys, int64_t d, MxOrder o, const float* weights,
                                                        OUT* y, int64_t ld_y, uint32_t spans) {
    const uint32_t group = blockIdx.x / spans, span = blockIdx.x - group * spans;
    const int64_t token = (int64_t)group * 4 + (threadIdx.x >> 6);
    if (token >= o.tokens) return;
    float acc[2][8] = {};
    // the rows of up to four choices are on their way at once; they are added in order
    constexpr int kAtOnce = 4;
    for (int j0 = 0; j0 < o.top_k; j0 += kAtOnce) {
        uint32_t slot[kAtOnce];
        float w[kAtOnce];
        Piece<IN, STREAM> rows[kAtOnce][2];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int64_t choice = token * o.top_k + j0 + j;
            slot[j] = j0 + j < o.top_k ? (uint32_t)o.slot_of[choice] : ~0u;
            w[j] = WEIGHTS && j0 + j < o.top_k ? weights[choice] : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c = (int64_t)span * kRowSpan + h * 512 + (threadIdx.x & 63) * 8;
                if (slot[j] < (uint32_t)o.capacity && c < d) rows[j][h].load(ys + slot[j] * ld_ys, c, d);
                else rows[j][h].clear();
            }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (slot[j] >= (uint32_t)o.capacity) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c = (int64_t)span * kRowSpan + h * 512 + (threadIdx.x & 63) * 8;
                float f[8];
                rows[j][h].values(c, d, f);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[h][i] += WEIGHTS ? w[j] * f[i] : f[i];
            }
        }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t c = (int64_t)span * kRowSpan + h * 512 + (threadIdx.x & 63) * 8;
        if (c < d) store_values<STREAM>(y + token * ld_y, c, d, acc[h]);
    }
}

// One wave per slot: the token's row is read for both gradients.  The lanes' partial sums, in binary32, are joined in a fixed order.
// Bound by memory (16384 of 18432 slots of 4096, both gradients: 65 us, 5.4 TB/s; of 2048, the weights' alone: 21 us, 4.8 TB/s).
template <class IN, bool DYS, bool DW, bool STREAM>
__global__ __launch_bounds__(256) void k_expert_combine_backward(const uint16_t* dy, int64_t ld_dy, const IN* ys, int64_t ld_ys, int64_t d,
                                                                 MxOrder o, const float* weights, uint16_t* dys, int64_t ld_dys, float* dweights) {
    const int64_t choices = (int64_t)o.tokens * o.top_k;
    if (DW) {                           // dropped choices have no slot: their zeros are shared out over all lanes
        const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
        if (i < choices && (uint32_t)o.slot_of[i] >= (uint32_t)o.capacity) dweights[i] = 0.0f;
    }
    const int64_t slot = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (slot >= o.capacity) return;
    const uint32_t choice = (uint32_t)o.src[slot];
    const bool used = choice < (uint64_t)choices;
    if (!used && !DYS) return;
    const uint16_t* row = used ? dy + (int64_t)(choice / (uint32_t)o.top_k) * ld_dy : nullptr;
    const float w = DYS && used ? weights[choice] : 0.0f;
    float sum = 0.0f;
    for (int64_t c = (threadIdx.x & 63) * 8; c < d; c += 512) {
        float g[8] = {};
        if (used) widen8(load8(row, c, d), g);
        if (DW && used) {
            Piece<IN, STREAM> piece;
            piece.load(ys + slot * ld_ys, c, d);
            float f[8];
            piece.values(c, d, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(g[i], f[i], sum);
        }
        if (DYS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] = used ? g[i] * w : 0.0f;
            store8<STREAM>(dys + slot * ld_dys, c, d, narrow8(g));
        }
    }
    if (DW && used) {
#pragma unroll
        for (int s = 32; s; s >>= 1) sum += __shfl_xor(sum, s);
        if ((threadIdx.x & 63) == 0) dweights[choice] = sum;
    }
}

uint32_t four_per_block(int64_t n) { return (uint32_t)((n + 3) / 4); }
uint32_t row_spans(int64_t d) { return (uint32_t)((d + kRowSpan - 1) / kRowSpan); }

}  // namespace

// Rounds of 1024 choices per workgroup, and workgroups.
static int sort_rounds(int64_t choices) {
    if (choices <= kSortLone) return (int)std::max<int64_t>((choices + kSortThreads - 1) / kSortThreads, 1);
    return (int)((choices + kSortChunks * kSortThreads - 1) / (kSortChunks * kSortThreads));
}
static int64_t sort_chunks(int64_t choices) {
    const int64_t each = (int64_t)sort_rounds(choices) * kSortThreads;
    return std::max<int64_t>((choices + each - 1) / each, 1);
}

size_t mx_sort_workspace(int64_t choices, int64_t n_experts) {
    const int64_t chunks = sort_chunks(choices);
    return chunks <= 1 ? 0 : (size_t)(chunks * n_experts * 4 + 15) / 16 * 16;
}

hipError_t launch_expert_sort(const int32_t* ids, const MxOrder& o, void* workspace, hipStream_t st) {
    const int64_t choices = (int64_t)o.tokens * o.top_k, chunks = sort_chunks(choices);
    const int rounds = sort_rounds(choices);
    if (chunks <= 1) {
        k_expert_place<true><<<dim3(1), dim3(kSortThreads), 0, st>>>(ids, choices, nullptr, o, rounds);
    } else {
        uint32_t* counts = static_cast<uint32_t*>(workspace);
        k_expert_count<<<dim3((uint32_t)chunks), dim3(kSortThreads), 0, st>>>(ids, choices, (uint32_t)o.n_experts, counts, rounds);
        k_expert_place<false><<<dim3((uint32_t)chunks), dim3(kSortThreads), 0, st>>>(ids, choices, counts, o, rounds);
    }
    return hipGetLastError();
}

hipError_t launch_expert_gather(const uint16_t* x, int64_t ld_x, int64_t d, const MxOrder& o, uint16_t* xs, int64_t ld_xs, hipStream_t st) {
    const uint32_t spans = row_spans(d);
    const int64_t blocks = (int64_t)four_per_block(o.capacity) * spans;
    if (blocks > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)blocks);
    if (mx_streamed(o.capacity * d, xs, ld_xs, 0)) k_expert_gather<true><<<grid, dim3(256), 0, st>>>(x, ld_x, d, o, xs, ld_xs, spans);
    else k_expert_gather<false><<<grid, dim3(256), 0, st>>>(x, ld_x, d, o, xs, ld_xs, spans);
    return hipGetLastError();
}

// (in elements of two bytes)
static bool streamed(int64_t elements, const uint16_t* rows, int64_t ld) { return mx_streamed(elements, rows, ld, 0); }
static bool streamed(int64_t elements, const float* rows, int64_t ld) { return mx_streamed(elements * 2, reinterpret_cast<const uint16_t*>(rows), ld * 2, 0); }

template <class IN, class OUT>
static hipError_t combine(const IN* ys, int64_t ld_ys, int64_t d, const MxOrder& o, const float* weights, OUT* y, int64_t ld_y, hipStream_t st) {
    const uint32_t spans = row_spans(d);
    const int64_t blocks = (int64_t)four_per_block(o.tokens) * spans;
    if (blocks > 0x7FFFFFFFll) return hipErrorInvalidValue;
    const dim3 grid((uint32_t)blocks);
    const bool stream = streamed(o.capacity * d, ys, ld_ys) && streamed(o.capacity * d, y, ld_y);
    if (weights) {
        if (stream) k_expert_combine<IN, OUT, true, true><<<grid, dim3(256), 0, st>>>(ys, ld_ys, d, o, weights, y, ld_y, spans);
        else k_expert_combine<IN, OUT, true, false><<<grid, dim3(256), 0, st>>>(ys, ld_ys, d, o, weights, y, ld_y, spans);
    } else {
        if (stream) k_expert_combine<IN, OUT, false, true><<<grid, dim3(256), 0, st>>>(ys, ld_ys, d, o, weights, y, ld_y, spans);
        else k_expert_combine<IN, OUT, false, false><<<grid, dim3(256), 0, st>>>(ys, ld_ys, d, o, weights, y, ld_y, spans);
    }
    return hipGetLastError();
}
hipError_t launch_expert_combine(const uint16_t* ys, int64_t ld_ys, int64_t d, const MxOrder& o, const float* weights, uint16_t* y,
                                 int64_t ld_y, hipStream_t st) {
    return combine(ys, ld_ys, d, o, weights, y, ld_y, st);
}
hipError_t launch_expert_combine_f32(const float* ys, int64_t ld_ys, int64_t d, const MxOrder& o, const float* weights, void* y, int64_t ld_y,
                                     bool y_f32, hipStream_t st) {
    return y_f32 ? combine(ys, ld_ys, d, o, weights, static_cast<float*>(y), ld_y, st) : combine(ys, ld_ys, d, o, weights, static_cast<uint16_t*>(y), ld_y, st);
}

template <class IN, bool STREAM>
static void combine_backward(const uint16_t* dy, int64_t ld_dy, const IN* ys, int64_t ld_ys, int64_t d, const MxOrder& o,
                             const float* weights, uint16_t* dys, int64_t ld_dys, float* dweights, hipStream_t st) {
    const dim3 grid(four_per_block(o.capacity));
    if (dys && dweights) k_expert_combine_backward<IN, true, true, STREAM><<<grid, dim3(256), 0, st>>>(dy, ld_dy, ys, ld_ys, d, o, weights, dys, ld_dys, dweights);
    else if (dweights) k_expert_combine_backward<IN, false, true, STREAM><<<grid, dim3(256), 0, st>>>(dy, ld_dy, ys, ld_ys, d, o, weights, dys, ld_dys, dweights);
    else                                // reads no rows, of whatever type
        k_expert_combine_backward<uint16_t, true, false, STREAM><<<grid, dim3(256), 0, st>>>(dy, ld_dy, nullptr, 0, d, o, weights, dys, ld_dys, dweights);
}
template <class IN>
static hipError_t backward(const uint16_t* dy, int64_t ld_dy, const IN* ys, int64_t ld_ys, int64_t d, const MxOrder& o, const float* weights,
                           uint16_t* dys, int64_t ld_dys, float* dweights, hipStream_t st) {
    if ((!ys || streamed(o.capacity * d, ys, ld_ys)) && (!dys || streamed(o.capacity * d, dys, ld_dys)))
        combine_backward<IN, true>(dy, ld_dy, ys, ld_ys, d, o, weights, dys, ld_dys, dweights, st);
    else combine_backward<IN, false>(dy, ld_dy, ys, ld_ys, d, o, weights, dys, ld_dys, dweights, st);
    return hipGetLastError();
}
hipError_t launch_expert_combine_backward(const uint16_t* dy, int64_t ld_dy, const uint16_t* ys, int64_t ld_ys, int64_t d, const MxOrder& o,
                                          const float* weights, uint16_t* dys, int64_t ld_dys, float* dweights, hipStream_t st) {
    return backward(dy, ld_dy, ys, ld_ys, d, o, weights, dys, ld_dys, dweights, st);
}
hipError_t launch_expert_combine_backward_f32(const uint16_t* dy, int64_t ld_dy, const float* ys, int64_t ld_ys, int64_t d, const MxOrder& o,
                                              const float* weights, uint16_t* dys, int64_t ld_dys, float* dweights, hipStream_t st) {
    return backward(dy, ld_dy, ys, ld_ys, d, o, weights, dys, ld_dys, dweights, st);
}

}  // namespace mor
