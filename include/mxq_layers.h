/*
 * mxq_layers.h -- the part of libmxq's C ABI that works on the layers of a language model around its
 * microscaled tensors: the norm in front of a projection (with the residual's addition and an output
 * in 8 bits with scales), projections over packed FP4 weights with the low-rank adapters of many
 * requests beside them, the gated activation between two projections, and the backward passes of norm
 * and activation from checkpoints that are kept in 8 bits.
 *
 * The 8-bit format, Q8.  A row is cut into blocks of 32 consecutive elements.  Each block has one scale
 * byte, S = 2^(byte-127) (E8M0), the smallest power of two with which no element exceeds 448 (bytes
 * below 0 are 0, so an all-zero block has byte 0), and one E4M3 byte per element, v / S rounded to
 * nearest even (OFP8: bias 7, largest value 448, 0x7F = NaN).  The largest element is never clipped,
 * and small elements beside an outlier keep three bits of mantissa down to 2^-15 of it.  A block with a
 * NaN or an infinity has scale byte 255: it reads back as NaN.  Codes are `rows x cols` bytes, scales
 * `rows x cols/32` bytes, row-major, contiguous.
 *
 * Conventions are those of mxq.h (device pointers of the caller, nothing allocated, work enqueued on
 * `stream`, status returned, every argument checked on the host first), with these additions
 *   - Dense inputs are `rows x cols` with a row stride in elements (`ld_...` >= cols), so halves of a
 *     wider tensor can be passed as they are.  Their base and every row are 16-byte aligned.  A stride
 *     of a tensor with at most one row is not looked at.
 *   - Dense outputs are contiguous unless a stride is listed.
 *   - NaN and infinities follow the formulas.  Sums are fp32.
 *   - rows == 0 or cols == 0 is a valid no-op, except where an output does not depend on rows.
 */
#ifndef MXQ_LAYERS_H
#define MXQ_LAYERS_H

#include "mxq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Elements that share a scale byte in Q8. */
#define MXQ_Q8_BLOCK 32

/* How mxq_linear may hold its sums. */
enum mxq_sums { MXQ_SUMS_F32 = 0, MXQ_SUMS_MX = 1 };

/* Longest row of mxq_add_rmsnorm and its backward pass. */
#define MXQ_NORM_MAX_COLS 16384

/*
 * mxq_add_rmsnorm -- t = x + residual; rstd = 1 / sqrt(mean(t^2) + eps); n = t * rstd; y = n * weight.
 * One launch, one pass over the inputs.  All of it in fp32; each output is rounded once.
 *
 *   x, residual   device, rows x cols of dtype; residual NULL: t = x
 *   weight        device, cols of dtype, 16-byte aligned; NULL: y = n
 *   cols          a multiple of 32, at most MXQ_NORM_MAX_COLS (UNSUPPORTED beyond)
 *   eps           finite, >= 0
 *   hidden_out    device, t in dtype, 16-byte aligned, or NULL.  May be the residual itself or x itself
 *                 (same base, contiguous): the residual stream is then updated in place.
 *   y_codes, y_scales   device, y as Q8, 8-byte and 1-byte aligned, or both NULL
 *   y_out         device, y in dtype, 16-byte aligned, or NULL
 *   n_codes, n_scales   device, n as Q8 (the checkpoint for the backward pass), or both NULL
 *   rstd_out      device, rows floats, 4-byte aligned, or NULL
 * At least one output must be given; none but hidden_out may overlap an input.
 */
MXQ_API int mxq_add_rmsnorm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* weight,
                            int64_t rows, int64_t cols, float eps, int dtype, void* hidden_out,
                            uint8_t* y_codes, uint8_t* y_scales, void* y_out,
                            uint8_t* n_codes, uint8_t* n_scales, float* rstd_out, void* stream);

/*
 * mxq_add_rmsnorm_backward -- the gradient of the above from the 8-bit checkpoint.  With n read back
 * from Q8 and g = dy * weight:
 *     dx      = rstd * (g - n * mean(g * n)) + dhidden     (the gradient of x and of the residual)
 *     dweight = sum over rows of dy * n
 * Two launches (one without dweight).  The sum over rows is formed in an order that depends on the
 * sizes alone: equal inputs give equal bits.
 *
 *   dy            device, gradient of y, rows x cols of dtype
 *   n_codes, n_scales, rstd   device, as written by mxq_add_rmsnorm
 *   weight        NULL: g = dy
 *   dhidden       device, gradient that reaches t by its other way (the residual stream), or NULL
 *   dx_out        device, rows x cols of dtype, contiguous, 16-byte aligned.  May be dy or dhidden
 *                 itself (same base, contiguous).
 *   dweight_out   device, cols floats, 4-byte aligned, or NULL.  Zeros when rows == 0.
 *   workspace     device, at least mxq_add_rmsnorm_backward_workspace_size(rows, cols) bytes, 16-byte
 *                 aligned; contents need no initial value; not looked at without dweight_out
 */
MXQ_API size_t mxq_add_rmsnorm_backward_workspace_size(int64_t rows, int64_t cols);
MXQ_API int mxq_add_rmsnorm_backward(const void* dy, int64_t ld_dy, const uint8_t* n_codes, const uint8_t* n_scales,
                                     const float* rstd, const void* weight, const void* dhidden, int64_t ld_dhidden,
                                     int64_t rows, int64_t cols, int dtype, void* dx_out, float* dweight_out,
                                     void* workspace, size_t workspace_bytes, void* stream);

/*
 * mxq_swiglu -- h = gate * sigmoid(gate) * up.
 *
 *   gate, up      device, rows x cols of dtype; cols a multiple of 32
 *   h_codes, h_scales   device, h as Q8, or both NULL
 *   h_out         device, h in dtype, 16-byte aligned, or NULL
 *   gate_codes .. up_scales   device, gate and up as Q8 (the checkpoint for the backward pass), or all NULL
 * At least one output must be given; none may overlap an input.
 */
MXQ_API int mxq_swiglu(const void* gate, int64_t ld_gate, const void* up, int64_t ld_up, int64_t rows, int64_t cols, int dtype,
                       uint8_t* h_codes, uint8_t* h_scales, void* h_out,
                       uint8_t* gate_codes, uint8_t* gate_scales, uint8_t* up_codes, uint8_t* up_scales, void* stream);

/*
 * mxq_swiglu_backward -- the gradients of gate and up from the 8-bit checkpoint.  With s = sigmoid(gate):
 *     dgate = dh * up * s * (1 + gate * (1 - s)),   dup = dh * gate * s
 * and, if asked for, h = gate * s * up once more (so that the forward pass need not keep it).
 *
 *   dgate_out, dup_out   device, rows x cols of dtype with row strides of their own, 16-byte aligned rows.
 *                 Either may be dh itself (same base, same stride).
 *   h_out         device, rows x cols of dtype, contiguous, 16-byte aligned, or NULL
 */
MXQ_API int mxq_swiglu_backward(const void* dh, int64_t ld_dh, const uint8_t* gate_codes, const uint8_t* gate_scales,
                                const uint8_t* up_codes, const uint8_t* up_scales, int64_t rows, int64_t cols, int dtype,
                                void* dgate_out, int64_t ld_dgate, void* dup_out, int64_t ld_dup, void* h_out, void* stream);

/*
 * mxq_linear -- a projection over weights as mxq_quantize packs them, with the low-rank adapters of
 * many requests beside it:
 *     y[i, :] = T * X[i, :] * W^T  +  scaling[a] * (X[i, :] * A[a]^T) * B[a]^T,   a = ids[i],
 * X the activations (m x k, bf16 or Q8), W[j, l] = q * S the packed weights (n x k), T their
 * per-tensor scale.  W is never unpacked in memory.  Products of elements are exact (bf16 holds q * S and
 * Q8's elements), sums are fp32, the adapters' inner product among them, y is rounded once.  With
 * MXQ_SUMS_MX, Q8 against E8M0 weights of block 32 and more, with a bf16 output, multiplies in the formats
 * themselves, up to twice as fast: the scaled matrix instruction sums 128 products with an error of up to
 * 2^-14 of their magnitudes (2^-18 where their sizes are alike) before it adds them in fp32.
 *
 *   x, ld_x       device, m x k bf16, rows 16-byte aligned; NULL if x_codes is given
 *   x_codes, x_scales   device, m x k as Q8, 16-byte and 1-byte aligned; NULL if x is given
 *   m, n, k       m, n at most 2^26; k below 2^22, a multiple of 32 and of block
 *   w_codes, w_scales   device, n x k as written by mxq_quantize, 16-byte and 4-byte aligned
 *   block         8 .. 128.  Blocks of 2 and 4 are UNSUPPORTED (more bits for scales than for codes, or as
 *                 many)
 *   tensor_scale  finite and > 0; not looked at if tensor_scale_dev is given
 *   tensor_scale_dev   device, the float that mxq_quantize_hier wrote, or NULL
 *   adapter_a, adapter_b   device, bf16, adapter_count x rank x k and adapter_count x n x rank, contiguous,
 *                 16-byte aligned; NULL: no adapters
 *   adapter_scaling   device, adapter_count floats
 *   adapter_ids   device, m int32: the adapter of each row.  A value outside 0 .. adapter_count-1 means
 *                 none.  NULL: every row takes adapter 0
 *   adapter_rank  8 .. 64, a multiple of 8
 *   sums          MXQ_SUMS_F32, or MXQ_SUMS_MX: the caller takes the sums of the scaled matrix instruction where
 *                 types, format and block allow it (elsewhere as MXQ_SUMS_F32)
 *   y, ld_y       device, m x n of y_dtype, row stride ld_y >= n, aligned to its elements; not
 *                 overlapping an input
 *   workspace     device, 16-byte aligned, at least mxq_linear_workspace_size(args) bytes (often 0); contents need
 *                 no initial value
 * k == 0 writes zeros.  Equal inputs give equal bits.  Rows do not mix: a NaN in one row of X or of W stays in that row or
 * column of y.  Like the rest of the library the call is re-entrant, workspaces aside.
 */
typedef struct mxq_linear_args {
    const void* x;
    int64_t ld_x;
    const uint8_t* x_codes;
    const uint8_t* x_scales;
    int64_t m, n, k;
    const uint8_t* w_codes;
    const uint8_t* w_scales;
    int block, scale_fmt;
    float tensor_scale;
    const float* tensor_scale_dev;
    const void* adapter_a;
    const void* adapter_b;
    const float* adapter_scaling;
    const int32_t* adapter_ids;
    int adapter_count, adapter_rank;
    void* y;
    int64_t ld_y;
    int y_dtype;
    void* workspace;
    size_t workspace_bytes;
    int sums;
} mxq_linear_args;
MXQ_API size_t mxq_linear_workspace_size(const mxq_linear_args* args);
MXQ_API int mxq_linear(const mxq_linear_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MXQ_LAYERS_H */
