// C ABI of the microscaled 4-bit operands and of tokens sorted by expert (mor_mx.h): argument validation and dispatch only.
#include "../../include/mor_mx.h"
#include "mx_launch.h"

namespace {

constexpr int64_t kMaxChoices = 1 << 24;
constexpr int64_t kMaxDim = 0x7FFFFFFF - 127;      // rows and columns: block and tile numbers fit 32 bits

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A packed operand with rows of `cols` elements.
mor_status check_operand(const mor_mx_operand* o, int64_t cols, bool batched) {
    if (!o || !o->codes || !o->scales) return MOR_ERR_NULL;
    const int64_t blocks = (cols + mor::kMxBlock - 1) / mor::kMxBlock;
    if (o->ld_codes < 16 * blocks || o->ld_scales < blocks) return MOR_ERR_SHAPE;
    if (o->ld_codes % 16 || o->ld_scales % 4 || !aligned(o->codes, 16) || !aligned(o->scales, 4)) return MOR_ERR_ALIGN;
    if (batched && (o->batch_codes % 16 || o->batch_scales % 4)) return MOR_ERR_ALIGN;
    if (batched && (o->batch_codes < 0 || o->batch_scales < 0)) return MOR_ERR_SHAPE;
    return MOR_OK;
}
mor::MxOperand operand_of(const mor_mx_operand* o, bool batched) {
    if (!o) return mor::MxOperand{nullptr, 0, nullptr, 0, 0, 0};
    return mor::MxOperand{o->codes, o->ld_codes, o->scales, o->ld_scales, batched ? o->batch_codes : 0, batched ? o->batch_scales : 0};
}

// A matrix of values of `size` bytes, whose rows may start at any of them.
mor_status check_matrix(const void* p, int64_t ld, int64_t cols, int size = 2) {
    if (!p) return MOR_ERR_NULL;
    if (ld < cols) return MOR_ERR_SHAPE;
    if (!aligned(p, size)) return MOR_ERR_ALIGN;
    return MOR_OK;
}

mor_status check_order(const mor_expert_order* o) {
    if (!o) return MOR_ERR_NULL;
    const int64_t need = mor_expert_capacity(o->tokens, o->top_k, o->n_experts, o->align);
    if (need < 0 || o->capacity < need || o->capacity % o->align || o->reserved != 0) return MOR_ERR_SHAPE;
    if (!o->offsets || (o->tokens > 0 && !o->slot_of) || (o->capacity > 0 && !o->src)) return MOR_ERR_NULL;
    if (!aligned(o->offsets, 4) || !aligned(o->slot_of, 4) || !aligned(o->src, 4)) return MOR_ERR_ALIGN;
    return MOR_OK;
}
mor_status check_combine(const void* ys, int64_t ld_ys, int ys_size, int64_t d, const mor_expert_order* order, const float* weights, const void* y,
                         int64_t ld_y, int y_size) {
    mor_status st = check_order(order);
    if (st != MOR_OK) return st;
    if (d < 1 || d > kMaxDim) return MOR_ERR_SHAPE;
    if (order->tokens == 0) return MOR_OK;
    if ((st = check_matrix(ys, ld_ys, d, ys_size)) != MOR_OK || (st = check_matrix(y, ld_y, d, y_size)) != MOR_OK) return st;
    return aligned(weights, 4) ? MOR_OK : MOR_ERR_ALIGN;
}
mor_status check_combine_backward(const uint16_t* dy, int64_t ld_dy, const void* ys, int64_t ld_ys, int ys_size, int64_t d,
                                  const mor_expert_order* order, const float* weights, const uint16_t* dys, int64_t ld_dys, const float* dweights) {
    mor_status st = check_order(order);
    if (st != MOR_OK) return st;
    if (d < 1 || d > kMaxDim) return MOR_ERR_SHAPE;
    if (order->capacity == 0) return MOR_OK;            // empty gradients have no address
    if (!dys && !dweights) return MOR_ERR_NULL;
    if (order->tokens > 0) {
        if ((st = check_matrix(dy, ld_dy, d)) != MOR_OK) return st;
        if (dweights && (st = check_matrix(ys, ld_ys, d, ys_size)) != MOR_OK) return st;
        if (dys && !weights) return MOR_ERR_NULL;
    }
    if (dys && (st = check_matrix(dys, ld_dys, d)) != MOR_OK) return st;
    return aligned(weights, 4) && aligned(dweights, 4) ? MOR_OK : MOR_ERR_ALIGN;
}
mor::MxOrder order_of(const mor_expert_order* o) {
    return mor::MxOrder{o->tokens, o->top_k, o->n_experts, o->align, o->capacity, o->offsets, o->slot_of, o->src};
}

mor_status launched(hipError_t e) { return e == hipSuccess ? MOR_OK : MOR_ERR_HIP; }

mor_status check_product(int64_t m, int64_t n, int64_t k, int32_t c_type) {
    if (m < 0 || n < 0 || k < 1 || m > kMaxDim || n > kMaxDim || k > kMaxDim) return MOR_ERR_SHAPE;
    if (c_type != MOR_MX_OUT_BF16 && c_type != MOR_MX_OUT_F32) return MOR_ERR_UNSUPPORTED;
    return MOR_OK;
}

mor::MxProductArgs product_args(int64_t m, int64_t n, int64_t k, const mor_mx_operand* a, const mor_mx_operand* b, void* c, int64_t ld_c,
                                int32_t c_type) {
    mor::MxProductArgs p{};
    p.a = a->codes; p.lda = a->ld_codes; p.as = a->scales; p.lda_s = a->ld_scales;
    p.b = b->codes; p.ldb = b->ld_codes; p.bs = b->scales; p.ldb_s = b->ld_scales;
    p.c = c; p.ldc = ld_c;
    p.m = m; p.n = n;
    p.blocks = (int32_t)((k + mor::kMxBlock - 1) / mor::kMxBlock);
    p.n_experts = 1;
    p.f32 = c_type == MOR_MX_OUT_F32;
    return p;
}

}  // namespace

extern "C" {

mor_status mor_mx_quantize(const mor_mx_params* p, const uint16_t* x, const mor_mx_operand* out, const mor_mx_operand* out_t,
                           const mor_expert_order* order, const float* weights, void* stream) {
    if (!p || (!out && !out_t)) return MOR_ERR_NULL;
    if (p->scale_rule != MOR_MX_SCALE_FLOOR && p->scale_rule != MOR_MX_SCALE_CEIL) return MOR_ERR_UNSUPPORTED;
    if (p->rounding != MOR_MX_ROUND_NEAREST && p->rounding != MOR_MX_ROUND_STOCHASTIC) return MOR_ERR_UNSUPPORTED;
    if (p->rows < 0 || p->cols < 1 || p->rows > kMaxDim || p->cols > kMaxDim || p->batch < 1 || p->batch > 65535) return MOR_ERR_SHAPE;
    const bool batched = p->batch > 1;
    if (batched && p->batch_x < 0) return MOR_ERR_SHAPE;
    int64_t rows = p->rows;
    mor_status st;
    if (order) {
        if (batched) return MOR_ERR_UNSUPPORTED;
        if ((st = check_order(order)) != MOR_OK) return st;
        if (order->tokens != p->rows) return MOR_ERR_SHAPE;
        rows = order->capacity;
    } else if (weights) return MOR_ERR_UNSUPPORTED;
    if (rows == 0) return MOR_OK;
    if (p->rows > 0 && (st = check_matrix(x, p->ld, p->cols)) != MOR_OK) return st;    // (slots without tokens: x has no address)
    if (!aligned(weights, 4)) return MOR_ERR_ALIGN;
    if (out && (st = check_operand(out, p->cols, batched)) != MOR_OK) return st;
    if (out_t && (st = check_operand(out_t, rows, batched)) != MOR_OK) return st;
    mor::MxQuantArgs a{};
    a.x = x; a.rows = rows; a.cols = p->cols; a.ld = p->ld; a.batch_x = batched ? p->batch_x : 0; a.batch = (int32_t)p->batch;
    if (order) {
        a.src = order->src;
        a.slot_of = order->slot_of;
        a.choices = (uint32_t)order->tokens * (uint32_t)order->top_k;
        a.top_k = (uint32_t)order->top_k;
        a.weights = weights;
    }
    a.ceil_rule = p->scale_rule == MOR_MX_SCALE_CEIL;
    a.stochastic = p->rounding == MOR_MX_ROUND_STOCHASTIC;
    a.seed = p->seed;
    a.out = operand_of(out, batched);
    a.out_t = operand_of(out_t, batched);
    return launched(mor::launch_mx_quantize(a, (hipStream_t)stream));
}

mor_status mor_mx_dequantize(int64_t rows, int64_t cols, int64_t batch, const mor_mx_operand* operand, uint16_t* y, int64_t ld_y,
                             int64_t batch_y, void* stream) {
    if (rows < 0 || cols < 1 || rows > kMaxDim || cols > kMaxDim || batch < 1 || batch > 65535) return MOR_ERR_SHAPE;
    if (rows == 0) return MOR_OK;
    mor_status st = check_operand(operand, cols, batch > 1);
    if (st != MOR_OK) return st;
    if ((st = check_matrix(y, ld_y, cols)) != MOR_OK) return st;
    if (batch > 1 && batch_y < 0) return MOR_ERR_SHAPE;
    return launched(mor::launch_mx_dequantize(rows, cols, batch, operand_of(operand, batch > 1), y, ld_y, batch_y, (hipStream_t)stream));
}

size_t mor_mx_product_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (check_product(m, n, k, MOR_MX_OUT_BF16) != MOR_OK || m == 0 || n == 0) return 0;
    return mor::mx_product_workspace(m, n, (k + mor::kMxBlock - 1) / mor::kMxBlock);
}

mor_status mor_mx_product(int64_t m, int64_t n, int64_t k, const mor_mx_operand* a, const mor_mx_operand* b, void* c, int64_t ld_c,
                          int32_t c_type, void* workspace, size_t workspace_bytes, void* stream) {
    mor_status st = check_product(m, n, k, c_type);
    if (st != MOR_OK) return st;
    if (m == 0 || n == 0) return MOR_OK;
    if ((st = check_operand(a, k, false)) != MOR_OK || (st = check_operand(b, k, false)) != MOR_OK) return st;
    if ((st = check_matrix(c, ld_c, n, c_type == MOR_MX_OUT_F32 ? 4 : 2)) != MOR_OK) return st;
    const size_t need = mor_mx_product_workspace_bytes(m, n, k);
    if (need && (!workspace || workspace_bytes < need)) return MOR_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return MOR_ERR_ALIGN;
    const mor::MxProductArgs p = product_args(m, n, k, a, b, c, ld_c, c_type);
    return launched(mor::launch_mx_product(mor::kMxDense, p, workspace, (hipStream_t)stream));
}

mor_status mor_mx_product_rows(int64_t n, int64_t k, const mor_mx_operand* a, const mor_mx_operand* b, const mor_expert_order* order,
                               void* c, int64_t ld_c, int32_t c_type, void* stream) {
    mor_status st = check_order(order);
    if (st != MOR_OK) return st;
    if ((st = check_product(order->capacity, n, k, c_type)) != MOR_OK) return st;
    if (order->capacity == 0 || n == 0) return MOR_OK;
    const bool batched = order->n_experts > 1;
    if ((st = check_operand(a, k, false)) != MOR_OK || (st = check_operand(b, k, batched)) != MOR_OK) return st;
    if ((st = check_matrix(c, ld_c, n, c_type == MOR_MX_OUT_F32 ? 4 : 2)) != MOR_OK) return st;
    mor::MxProductArgs p = product_args(order->capacity, n, k, a, b, c, ld_c, c_type);
    p.batch_b = batched ? b->batch_codes : 0;
    p.batch_bs = batched ? b->batch_scales : 0;
    p.offsets = order->offsets;
    p.n_experts = order->n_experts;
    p.choices = order->tokens * order->top_k;
    p.align = order->align;
    return launched(mor::launch_mx_product(mor::kMxRows, p, nullptr, (hipStream_t)stream));
}

mor_status mor_mx_product_depth(int64_t m, int64_t n, const mor_mx_operand* a, const mor_mx_operand* b, const mor_expert_order* order,
                                void* c, int64_t ld_c, int64_t batch_c, int32_t c_type, void* stream) {
    mor_status st = check_order(order);
    if (st != MOR_OK) return st;
    if ((st = check_product(m, n, order->capacity > 0 ? order->capacity : 1, c_type)) != MOR_OK) return st;
    if (order->align % 128) return MOR_ERR_UNSUPPORTED;        // segments are whole steps of the product
    if (m == 0 || n == 0) return MOR_OK;
    if (!a || !b) return MOR_ERR_NULL;
    if (order->capacity > 0 &&                                 // without a slot the results are zeros and nothing is read
        ((st = check_operand(a, order->capacity, false)) != MOR_OK || (st = check_operand(b, order->capacity, false)) != MOR_OK)) return st;
    if ((st = check_matrix(c, ld_c, n, c_type == MOR_MX_OUT_F32 ? 4 : 2)) != MOR_OK) return st;
    if (order->n_experts > 1 && batch_c < 0) return MOR_ERR_SHAPE;
    mor::MxProductArgs p = product_args(m, n, order->capacity, a, b, c, ld_c, c_type);
    p.batch_c = order->n_experts > 1 ? batch_c : 0;
    p.offsets = order->offsets;
    p.n_experts = order->n_experts;
    return launched(mor::launch_mx_product(mor::kMxDepth, p, nullptr, (hipStream_t)stream));
}

int64_t mor_expert_capacity(int64_t tokens, int64_t top_k, int64_t n_experts, int64_t align) {
    if (tokens < 0 || top_k < 1 || top_k > kMaxChoices || tokens > kMaxChoices || tokens * top_k > kMaxChoices) return -1;
    if (n_experts < 1 || n_experts > MOR_EXPERTS_MAX || align < 1 || align > 65536) return -1;
    const int64_t choices = tokens * top_k;
    const int64_t most = choices + (choices < n_experts ? choices : n_experts) * (align - 1);
    return (most + align - 1) / align * align;
}
size_t mor_expert_workspace_bytes(int64_t tokens, int64_t top_k, int64_t n_experts) {
    if (mor_expert_capacity(tokens, top_k, n_experts, 1) < 0) return 0;
    return mor::mx_sort_workspace(tokens * top_k, n_experts);
}

mor_status mor_expert_sort(const int32_t* ids, const mor_expert_order* order, void* workspace, size_t workspace_bytes, void* stream) {
    const mor_status st = check_order(order);
    if (st != MOR_OK) return st;
    if (!ids && order->tokens > 0) return MOR_ERR_NULL;
    if (!aligned(ids, 4)) return MOR_ERR_ALIGN;
    const size_t need = mor_expert_workspace_bytes(order->tokens, order->top_k, order->n_experts);
    if (need && (!workspace || workspace_bytes < need)) return MOR_ERR_WORKSPACE;
    if (need && !aligned(workspace, 16)) return MOR_ERR_ALIGN;
    return launched(mor::launch_expert_sort(ids, order_of(order), workspace, (hipStream_t)stream));
}

mor_status mor_expert_gather(const uint16_t* x, int64_t ld_x, int64_t d, const mor_expert_order* order, uint16_t* xs, int64_t ld_xs,
                             void* stream) {
    mor_status st = check_order(order);
    if (st != MOR_OK) return st;
    if (d < 1 || d > kMaxDim) return MOR_ERR_SHAPE;
    if (order->capacity == 0) return MOR_OK;
    if (order->tokens > 0 && (st = check_matrix(x, ld_x, d)) != MOR_OK) return st;
    if ((st = check_matrix(xs, ld_xs, d)) != MOR_OK) return st;
    return launched(mor::launch_expert_gather(x, ld_x, d, order_of(order), xs, ld_xs, (hipStream_t)stream));
}

mor_status mor_expert_combine(const uint16_t* ys, int64_t ld_ys, int64_t d, const mor_expert_order* order, const float* weights,
                              uint16_t* y, int64_t ld_y, void* stream) {
    const mor_status st = check_combine(ys, ld_ys, 2, d, order, weights, y, ld_y, 2);
    if (st != MOR_OK || order->tokens == 0) return st;
    return launched(mor::launch_expert_combine(ys, ld_ys, d, order_of(order), weights, y, ld_y, (hipStream_t)stream));
}

mor_status mor_expert_combine_f32(const float* ys, int64_t ld_ys, int64_t d, const mor_expert_order* order, const float* weights, void* y,
                                  int64_t ld_y, int32_t y_type, void* stream) {
    if (y_type != MOR_MX_OUT_BF16 && y_type != MOR_MX_OUT_F32) return MOR_ERR_UNSUPPORTED;
    const bool y_f32 = y_type == MOR_MX_OUT_F32;
    const mor_status st = check_combine(ys, ld_ys, 4, d, order, weights, y, ld_y, y_f32 ? 4 : 2);
    if (st != MOR_OK || order->tokens == 0) return st;
    return launched(mor::launch_expert_combine_f32(ys, ld_ys, d, order_of(order), weights, y, ld_y, y_f32, (hipStream_t)stream));
}

mor_status mor_expert_combine_backward(const uint16_t* dy, int64_t ld_dy, const uint16_t* ys, int64_t ld_ys, int64_t d,
                                       const mor_expert_order* order, const float* weights, uint16_t* dys, int64_t ld_dys,
                                       float* dweights, void* stream) {
    const mor_status st = check_combine_backward(dy, ld_dy, ys, ld_ys, 2, d, order, weights, dys, ld_dys, dweights);
    if (st != MOR_OK || order->capacity == 0) return st;
    return launched(mor::launch_expert_combine_backward(dy, ld_dy, ys, ld_ys, d, order_of(order), weights, dys, ld_dys, dweights, (hipStream_t)stream));
}

mor_status mor_expert_combine_backward_f32(const uint16_t* dy, int64_t ld_dy, const float* ys, int64_t ld_ys, int64_t d,
                                           const mor_expert_order* order, const float* weights, uint16_t* dys, int64_t ld_dys,
                                           float* dweights, void* stream) {
    const mor_status st = check_combine_backward(dy, ld_dy, ys, ld_ys, 4, d, order, weights, dys, ld_dys, dweights);
    if (st != MOR_OK || order->capacity == 0) return st;
    return launched(mor::launch_expert_combine_backward_f32(dy, ld_dy, ys, ld_ys, d, order_of(order), weights, dys, ld_dys, dweights, (hipStream_t)stream));
}

}  // extern "C"
