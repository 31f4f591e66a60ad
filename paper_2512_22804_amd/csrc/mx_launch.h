// Host-side launch interface between the C ABI of the microscaled 4-bit operands (mx_api.hip) and their kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace mor {

constexpr int kMxBlock = 32;            // elements per scale

// Large tensors are read and written past the caches (non-temporal): they leave nothing behind that the next call could use.  Only rows
// of whole lines, since parts of a line that go past the caches one by one are slower.  (De-quantisation of 14336 x 4096: 21.3 us
// past the caches, 31.5 through them; of 18432 x 4104 40.4 and 28.2; of 4099 x 5001, which stays in the Infinity Cache, 14.1 and 12.8.)
constexpr int64_t kMxStreamBytes = 1 << 26;
constexpr int64_t kMxStreamReadBytes = 1 << 24;        // where only reads go past them (4096 x 4096 transposed: 11.1 us, 10.4 so)
inline bool mx_streamed(int64_t elements, const uint16_t* rows, int64_t ld, int64_t batch, int64_t least = kMxStreamBytes) {
    return elements * 2 >= least && ((reinterpret_cast<uintptr_t>(rows) | (uintptr_t)(ld * 2) | (uintptr_t)(batch * 2)) & 127) == 0;
}

// A packed operand on the device: codes and E8M0 bytes, leading dimensions and batch distances in bytes.
struct MxOperand {
    uint8_t* codes;  int64_t ld;
    uint8_t* scales; int64_t ld_s;
    int64_t  batch, batch_s;
};

// The order of tokens by expert, as the kernels see it.
struct MxOrder {
    int32_t  tokens, top_k, n_experts, align, capacity;
    int32_t* offsets;
    int32_t* slot_of;
    int32_t* src;
};

struct MxQuantArgs {
    const uint16_t* x;
    int64_t  rows, cols, ld, batch_x;   // rows of the output (slots when `src` is set)
    int32_t  batch;
    const int32_t* src;                 // choice of each row, or nullptr: row r of x is row r
    const int32_t* slot_of;             // slot of each choice (with `src`)
    uint32_t choices, top_k;
    const float* weights;               // factor of each choice, or nullptr
    int      ceil_rule;
    int      stochastic;
    uint64_t seed;
    MxOperand out, out_t;               // codes == nullptr: form not wanted
};
hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t st);
hipError_t launch_mx_dequantize(int64_t rows, int64_t cols, int64_t batch, const MxOperand& op, uint16_t* y, int64_t ld_y, int64_t batch_y,
                                hipStream_t st);

// Products: which rows and which depth a workgroup's tile covers.
enum { kMxDense = 0,      // one product
       kMxRows = 1,       // rows of A and C: the segment of an expert; B: that expert's operand of the batch
       kMxDepth = 2 };    // depth: the segment of an expert; C: that expert's result
struct MxProductArgs {
    const uint8_t* a;  int64_t lda;  const uint8_t* as; int64_t lda_s;
    const uint8_t* b;  int64_t ldb;  const uint8_t* bs; int64_t ldb_s;
    int64_t  batch_b, batch_bs;         // bytes between the experts' B (kMxRows)
    void*    c;        int64_t ldc, batch_c;   // elements
    int64_t  m, n;
    int32_t  blocks;                    // blocks of 32 along the depth
    const int32_t* offsets;             // experts' segments (kMxRows, kMxDepth)
    int32_t  n_experts;
    int32_t  choices, align;            // of the order: how many tiles to expect (kMxRows)
    int32_t  f32;                       // C in binary32, else BF16
    int32_t  splits;                    // (launcher) kMxDense: parts of the depth, each with a C of its own, batch_c apart
    int32_t  c_words;                   // (launcher) rows of C are whole 4-byte words and near each other
    int32_t  c_lines;                   // and of whole lines of 128 bytes
};
size_t mx_product_workspace(int64_t m, int64_t n, int32_t blocks);
hipError_t launch_mx_product(int mode, MxProductArgs p, void* workspace, hipStream_t st);

size_t mx_sort_workspace(int64_t choices, int64_t n_experts);
hipError_t launch_expert_sort(const int32_t* ids, const MxOrder& o, void* workspace, hipStream_t st);
hipError_t launch_expert_gather(const uint16_t* x, int64_t ld_x, int64_t d, const MxOrder& o, uint16_t* xs, int64_t ld_xs, hipStream_t st);
hipError_t launch_expert_combine(const uint16_t* ys, int64_t ld_ys, int64_t d, const MxOrder& o, const float* weights, uint16_t* y,
                                 int64_t ld_y, hipStream_t st);
hipError_t launch_expert_combine_f32(const float* ys, int64_t ld_ys, int64_t d, const MxOrder& o, const float* weights, void* y, int64_t ld_y,
                                     bool y_f32, hipStream_t st);
hipError_t launch_expert_combine_backward(const uint16_t* dy, int64_t ld_dy, const uint16_t* ys, int64_t ld_ys, int64_t d, const MxOrder& o,
                                          const float* weights, uint16_t* dys, int64_t ld_dys, float* dweights, hipStream_t st);
hipError_t launch_expert_combine_backward_f32(const uint16_t* dy, int64_t ld_dy, const float* ys, int64_t ld_ys, int64_t d, const MxOrder& o,
                                              const float* weights, uint16_t* dys, int64_t ld_dys, float* dweights, hipStream_t st);

}  // namespace mor
