/*
 * mor_mx.h -- C ABI of the microscaled 4-bit operands of the MI355X (gfx950) MoR library, of their products, and of
 * the sorting of tokens by expert that those products serve.  Same library, same conventions and status codes as
 * mor.h: device pointers owned by the caller, work enqueued on `stream`, nothing allocated or synchronized, argument
 * errors returned before anything is launched.
 *
 * A 4-bit operand [rows x cols] holds blocks of 32 consecutive elements of a row (the last block of a row may be
 * shorter; the elements that it lacks are stored as code 0).  It consists of
 *   codes   [rows x ld_codes] bytes, two E2M1 codes per byte, the element of even index in the low half:
 *           0, 0.5, 1, 1.5, 2, 3, 4, 6 for codes 0..7, bit 3 the sign; ceil(cols/32) * 16 bytes of a row are used
 *   scales  [rows x ld_scales] bytes, one E8M0 byte b per block: the elements stand for code * 2^(b - 127);
 *           b = 255: the block held an infinity or a NaN and stands for 32 NaNs
 * The scale 2^e of a block follows from its amax (largest magnitude): amax = 0: e = 0; otherwise the rule of
 * mor_mx_params, kept within [-127, 127].  The elements are rounded to the nearest value of the grid (ties to the
 * even code) or stochastically, magnitudes above 6 become 6, the sign is kept (also of zeros).
 *
 * Matrices of BF16 or binary32 values may have any leading dimension (in elements) from their row length on and need the
 * alignment of their elements only; 16-byte rows are read and written in whole pieces and are faster.
 *
 * The product of two operands sums over their columns, C = A B^T, so both hold their blocks along the depth.  The
 * products of a linear layer y = x W^T then read: forward: x and W; gradient of x: dy and W^T; gradient of W: dy^T and
 * x^T.  mor_mx_quantize writes an operand, its transpose, or both, from one read of the BF16 tensor.
 */
#ifndef MOR_MX_H_
#define MOR_MX_H_

#include "mor.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MOR_MX_SCALE_FLOOR = 0,  /* e = floor(log2(amax)) - 2: magnitudes in (6, 8) * 2^e are clipped to 6 * 2^e */
    MOR_MX_SCALE_CEIL = 1    /* the smallest e with amax <= 6 * 2^e: nothing is clipped */
} mor_mx_scale_rule;

typedef enum {
    MOR_MX_ROUND_NEAREST = 0,
    MOR_MX_ROUND_STOCHASTIC = 1  /* up with the probability of the distance to the lower neighbour, in 1/65536.  The 16
                                    random bits r of element (row, col) of an output form come from the counter-based
                                    generator Philox 4x32 with 7 rounds: counter (col / 8, row, batch, form), form 0 =
                                    rows, 1 = transposed, key (seed low, seed high), half (col % 2) of word
                                    (col % 8) / 2; the element becomes step * floor(|x| 2^-e / step + r / 65536), step
                                    being the distance of the grid's values around it */
} mor_mx_rounding;

typedef struct mor_mx_operand {
    uint8_t* codes;        /* 16-byte aligned */
    int64_t  ld_codes;     /* bytes, multiple of 16, >= 16 * ceil(cols / 32) */
    uint8_t* scales;       /* 4-byte aligned */
    int64_t  ld_scales;    /* bytes, multiple of 4, >= ceil(cols / 32); a product reads a row's bytes up to the next multiple of 4,
                              whatever stands there */
    int64_t  batch_codes;  /* bytes between the operands of a batch, multiple of 16 (ignored for one operand) */
    int64_t  batch_scales; /* the same of the scales, multiple of 4 */
} mor_mx_operand;

/* The order of tokens by expert that mor_expert_sort writes and the other calls read.  A choice i = t * top_k + j is the
 * j-th expert of token t.  The choices of one expert take consecutive slots in the order of i (the sort is stable); an
 * expert's first slot offsets[e] is a multiple of `align`, and slots between its last choice and offsets[e + 1] are
 * empty, as are all from offsets[n_experts] up to `capacity`. */
typedef struct mor_expert_order {
    int32_t  tokens, top_k, n_experts, align;  /* align in [1, 65536]; tokens * top_k <= 2^24; n_experts in [1, MOR_EXPERTS_MAX] */
    int32_t  capacity;       /* slots, >= mor_expert_capacity(...) and a multiple of align */
    int32_t  reserved;
    int32_t* offsets;        /* device [n_experts + 1] */
    int32_t* slot_of;        /* device [tokens * top_k]: slot of each choice, -1: dropped */
    int32_t* src;            /* device [capacity]: choice in each slot, -1: empty */
} mor_expert_order;
#define MOR_EXPERTS_MAX 1024

typedef struct mor_mx_params {
    int64_t  rows, cols, ld;  /* x: rows >= 0, cols >= 1; ld in elements, >= cols */
    int64_t  batch;           /* operands in one call, 1..65535 */
    int64_t  batch_x;         /* elements between them (ignored for one) */
    int32_t  scale_rule;      /* mor_mx_scale_rule */
    int32_t  rounding;        /* mor_mx_rounding */
    uint64_t seed;            /* stochastic rounding only */
} mor_mx_params;

/*
 * Quantises x (BF16 bit patterns).  out [rows x cols] and / or out_t [cols x rows] (NULL: not wanted, one
 * of them is): the transpose has its blocks along x's rows, shared by nothing with the blocks of `out`.
 * With `order` (batch 1) x holds the rows of order->tokens tokens (params->rows) and the operands have order->capacity
 * rows (out_t: columns): slot s holds the row of its choice's token, times weights[choice] in binary32 when `weights`
 * (device [tokens x top_k]) is given, and zeros where it is empty.
 */
mor_status mor_mx_quantize(const mor_mx_params* params, const uint16_t* x, const mor_mx_operand* out, const mor_mx_operand* out_t,
                           const mor_expert_order* order, const float* weights, void* stream);

/* y = what the operand stands for, in BF16 (exact; magnitudes from 2^-128 to 6 * 2^126, larger ones become infinite).
 * y: [rows x ld_y], ld_y and batch_y in elements. */
mor_status mor_mx_dequantize(int64_t rows, int64_t cols, int64_t batch, const mor_mx_operand* operand, uint16_t* y, int64_t ld_y,
                             int64_t batch_y, void* stream);

typedef enum { MOR_MX_OUT_BF16 = 0, MOR_MX_OUT_F32 = 1 } mor_mx_out;

/*
 * C [m x n] = A [m x k] B [n x k]^T, sums in binary32, rounded once to c_type.  ld_c in elements.
 * m or n = 0: nothing is done.  workspace: mor_mx_product_workspace_bytes(m, n, k) bytes of device scratch,
 * 16-byte aligned (may be NULL when that is 0); products that overlap in time must not share it.
 */
size_t     mor_mx_product_workspace_bytes(int64_t m, int64_t n, int64_t k);
mor_status mor_mx_product(int64_t m, int64_t n, int64_t k, const mor_mx_operand* a, const mor_mx_operand* b, void* c, int64_t ld_c,
                          int32_t c_type, void* workspace, size_t workspace_bytes, void* stream);

/*
 * One product per expert over its rows: rows offsets[e] .. offsets[e + 1] - 1 of C [capacity x n] are those rows of
 * A [capacity x k] times B_e [n x k]^T (the e-th operand of the batch `b`).  Rows from offsets[n_experts] on are left as
 * they are.
 */
mor_status mor_mx_product_rows(int64_t n, int64_t k, const mor_mx_operand* a, const mor_mx_operand* b, const mor_expert_order* order,
                               void* c, int64_t ld_c, int32_t c_type, void* stream);

/*
 * One product per expert over the depth that its slots are: C_e [m x n] = A [m x capacity] B [n x capacity]^T summed over
 * the columns offsets[e] .. offsets[e + 1] - 1 (zeros for an expert without any).  order->align must be a multiple of
 * 128.  batch_c: elements between the experts' results.
 */
mor_status mor_mx_product_depth(int64_t m, int64_t n, const mor_mx_operand* a, const mor_mx_operand* b, const mor_expert_order* order,
                                void* c, int64_t ld_c, int64_t batch_c, int32_t c_type, void* stream);

/* Smallest capacity that holds every order of these sizes, a multiple of align; -1 for invalid sizes. */
int64_t mor_expert_capacity(int64_t tokens, int64_t top_k, int64_t n_experts, int64_t align);
size_t  mor_expert_workspace_bytes(int64_t tokens, int64_t top_k, int64_t n_experts);

/* Sorts the choices: ids [tokens x top_k] holds the expert of each; one outside [0, n_experts) drops the choice.  Writes
 * order->offsets, slot_of and src (all of it).  workspace: mor_expert_workspace_bytes(...) bytes, 16-byte aligned. */
mor_status mor_expert_sort(const int32_t* ids, const mor_expert_order* order, void* workspace, size_t workspace_bytes, void* stream);

/* xs [capacity x d]: the row of x [tokens x d] for each slot, zeros for an empty one.  BF16. */
mor_status mor_expert_gather(const uint16_t* x, int64_t ld_x, int64_t d, const mor_expert_order* order, uint16_t* xs, int64_t ld_xs,
                             void* stream);

/* y [tokens x d] = sum over j of weights[t, j] * ys[slot of (t, j)], in the order of j, in binary32, rounded once to BF16;
 * weights NULL: all 1 (the gradient of mor_expert_gather).  Dropped choices add nothing; a token without any gets zeros. */
mor_status mor_expert_combine(const uint16_t* ys, int64_t ld_ys, int64_t d, const mor_expert_order* order, const float* weights,
                              uint16_t* y, int64_t ld_y, void* stream);

/* The same of rows in binary32, as mor_mx_product_rows writes them too: no rounding between the product and the sum.  y: BF16 or binary32. */
mor_status mor_expert_combine_f32(const float* ys, int64_t ld_ys, int64_t d, const mor_expert_order* order, const float* weights, void* y,
                                  int64_t ld_y, int32_t y_type, void* stream);

/* The gradients of mor_expert_combine with weights: dys [capacity x d] = weights[choice] * dy[its token] (zeros in empty slots) and
 * dweights [tokens x top_k] = <dy[t], ys[slot]> in binary32 (0 for a dropped choice).  Either may be NULL; ys is read for
 * dweights only, weights for dys only. */
mor_status mor_expert_combine_backward(const uint16_t* dy, int64_t ld_dy, const uint16_t* ys, int64_t ld_ys, int64_t d,
                                       const mor_expert_order* order, const float* weights, uint16_t* dys, int64_t ld_dys,
                                       float* dweights, void* stream);
/* The same of rows ys in binary32; dys stays BF16. */
mor_status mor_expert_combine_backward_f32(const uint16_t* dy, int64_t ld_dy, const float* ys, int64_t ld_ys, int64_t d,
                                           const mor_expert_order* order, const float* weights, uint16_t* dys, int64_t ld_dys,
                                           float* dweights, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOR_MX_H_ */
