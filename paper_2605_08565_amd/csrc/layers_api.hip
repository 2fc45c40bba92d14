// C ABI of the layer operators (see include/mxq_layers.h): host-side validation and dispatch.  No allocation, no
// synchronisation, no global state.
#include "../../include/mxq_layers.h"
#include "mxq_layers_launch.hpp"

#include <cmath>
#include <cstddef>
#include <cstdint>

namespace {

constexpr int64_t kMostElements = (int64_t)1 << 42;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int size_of(int dtype) { return dtype == MXQ_DT_BF16 ? 2 : 4; }

// Shape and type shared by the elementwise operators.
int check_shape(int64_t rows, int64_t cols, int dtype)
{
    if (rows < 0 || cols < 0 || cols % MXQ_Q8_BLOCK != 0) return MXQ_ERR_INVALID_ARG;
    if (dtype != MXQ_DT_BF16 && dtype != MXQ_DT_F32) return MXQ_ERR_INVALID_ARG;
    if (rows > 0 && cols > INT64_MAX / rows) return MXQ_ERR_INVALID_ARG;
    if (rows * cols >= kMostElements) return MXQ_ERR_UNSUPPORTED;
    return MXQ_OK;
}

// A dense tensor with a row stride: the stride holds a row, and every row starts on 16 bytes.
int check_rows(const void* p, int64_t ld, int64_t rows, int64_t cols, int dtype)
{
    if (rows > 1 && (ld < cols || ld > INT64_MAX / 8 / rows)) return MXQ_ERR_INVALID_ARG;
    if (!aligned(p, 16) || (rows > 1 && ld * size_of(dtype) % 16 != 0)) return MXQ_ERR_ALIGNMENT;
    return MXQ_OK;
}

// Codes and scales come together.
bool half_given(const void* codes, const void* scales) { return (codes == nullptr) != (scales == nullptr); }

int status(hipError_t e) { return e == hipSuccess ? MXQ_OK : MXQ_ERR_HIP; }

#define MXQ_TRY(call) do { const int s_ = (call); if (s_ != MXQ_OK) return s_; } while (0)

constexpr int64_t kMostSide = (int64_t)1 << 26;               // a grid counts 32-bit work items

mxq::LinearArgs linear_of(const mxq_linear_args& g)
{
    const bool adapters = g.adapter_a != nullptr;
    return {g.x, g.ld_x, g.x_codes, g.x_scales, (int)g.m, (int)g.n, (int)g.k, g.w_codes, g.w_scales, g.block, g.scale_fmt,
            g.tensor_scale, g.tensor_scale_dev, static_cast<const uint16_t*>(g.adapter_a), static_cast<const uint16_t*>(g.adapter_b),
            g.adapter_scaling, g.adapter_ids, adapters ? g.adapter_count : 0, adapters ? g.adapter_rank : 0, g.y, g.ld_y, g.y_dtype,
            g.sums == MXQ_SUMS_MX, nullptr, 0, 0, 0, nullptr, 1, 0};
}

// Everything that the sizes of workspace and launch depend on.
int check_linear(const mxq_linear_args& g)
{
    if (g.m < 0 || g.n < 0 || g.k < 0) return MXQ_ERR_INVALID_ARG;
    if (g.block < 2 || g.block > 128 || (g.block & (g.block - 1)) != 0) return MXQ_ERR_INVALID_ARG;
    if (g.k % MXQ_Q8_BLOCK != 0 || g.k % g.block != 0) return MXQ_ERR_INVALID_ARG;
    if (g.scale_fmt < MXQ_SCALE_E8M0 || g.scale_fmt > MXQ_SCALE_UE5M3) return MXQ_ERR_INVALID_ARG;
    if (g.y_dtype != MXQ_DT_BF16 && g.y_dtype != MXQ_DT_F32) return MXQ_ERR_INVALID_ARG;
    if (g.sums != MXQ_SUMS_F32 && g.sums != MXQ_SUMS_MX) return MXQ_ERR_INVALID_ARG;
    if ((g.adapter_a == nullptr) != (g.adapter_b == nullptr)) return MXQ_ERR_INVALID_ARG;
    if (g.adapter_a) {
        if (!g.adapter_scaling || g.adapter_count < 1) return MXQ_ERR_INVALID_ARG;
        if (g.adapter_rank < 8 || g.adapter_rank > 64 || g.adapter_rank % 8 != 0) return MXQ_ERR_INVALID_ARG;
    }
    if (g.block < 8 || g.m > kMostSide || g.n > kMostSide || g.k >= (1 << 22)) return MXQ_ERR_UNSUPPORTED;
    return MXQ_OK;
}

}  // namespace

extern "C" {

int mxq_add_rmsnorm(const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const void* weight,
                    int64_t rows, int64_t cols, float eps, int dtype, void* hidden_out,
                    uint8_t* y_codes, uint8_t* y_scales, void* y_out,
                    uint8_t* n_codes, uint8_t* n_scales, float* rstd_out, void* stream)
{
    MXQ_TRY(check_shape(rows, cols, dtype));
    if (!(eps >= 0.0f) || std::isinf(eps)) return MXQ_ERR_INVALID_ARG;
    if (half_given(y_codes, y_scales) || half_given(n_codes, n_scales)) return MXQ_ERR_INVALID_ARG;
    if (cols > MXQ_NORM_MAX_COLS) return MXQ_ERR_UNSUPPORTED;
    if (rows * cols == 0) return MXQ_OK;
    if (!x || !(hidden_out || y_codes || y_out || n_codes || rstd_out)) return MXQ_ERR_INVALID_ARG;
    MXQ_TRY(check_rows(x, ld_x, rows, cols, dtype));
    if (residual) MXQ_TRY(check_rows(residual, ld_residual, rows, cols, dtype));
    if (!aligned(weight, 16) || !aligned(hidden_out, 16) || !aligned(y_codes, 8) || !aligned(y_out, 16) || !aligned(n_codes, 8) ||
        !aligned(rstd_out, 4))
        return MXQ_ERR_ALIGNMENT;
    const mxq::NormArgs a = {x, residual, weight, ld_x, ld_residual, rows, (int)cols, eps, hidden_out, y_codes, y_scales, y_out,
                             n_codes, n_scales, rstd_out};
    return status(mxq::launch_add_rmsnorm(a, dtype, static_cast<hipStream_t>(stream)));
}

size_t mxq_add_rmsnorm_backward_workspace_size(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || cols > MXQ_NORM_MAX_COLS) return 0;
    return (size_t)mxq::norm_back_groups(rows, cols) * (size_t)cols * sizeof(float);
}

int mxq_add_rmsnorm_backward(const void* dy, int64_t ld_dy, const uint8_t* n_codes, const uint8_t* n_scales,
                             const float* rstd, const void* weight, const void* dhidden, int64_t ld_dhidden,
                             int64_t rows, int64_t cols, int dtype, void* dx_out, float* dweight_out,
                             void* workspace, size_t workspace_bytes, void* stream)
{
    MXQ_TRY(check_shape(rows, cols, dtype));
    if (cols > MXQ_NORM_MAX_COLS) return MXQ_ERR_UNSUPPORTED;
    if (cols == 0 || (rows == 0 && !dweight_out)) return MXQ_OK;
    if (rows > 0) {
        if (!dy || !n_codes || !n_scales || !rstd || !dx_out) return MXQ_ERR_INVALID_ARG;
        if (dweight_out && (!workspace || workspace_bytes < mxq_add_rmsnorm_backward_workspace_size(rows, cols))) return MXQ_ERR_INVALID_ARG;
        MXQ_TRY(check_rows(dy, ld_dy, rows, cols, dtype));
        if (dhidden) MXQ_TRY(check_rows(dhidden, ld_dhidden, rows, cols, dtype));
        if (!aligned(n_codes, 8) || !aligned(rstd, 4) || !aligned(weight, 16) || !aligned(dx_out, 16) ||
            (dweight_out && !aligned(workspace, 16)))
            return MXQ_ERR_ALIGNMENT;
    }
    if (!aligned(dweight_out, 4)) return MXQ_ERR_ALIGNMENT;
    const mxq::NormBackArgs a = {dy, n_codes, n_scales, rstd, weight, dhidden, ld_dy, ld_dhidden, rows, (int)cols, dx_out, dweight_out,
                                 static_cast<float*>(workspace)};
    return status(mxq::launch_add_rmsnorm_backward(a, dtype, static_cast<hipStream_t>(stream)));
}

int mxq_swiglu(const void* gate, int64_t ld_gate, const void* up, int64_t ld_up, int64_t rows, int64_t cols, int dtype,
               uint8_t* h_codes, uint8_t* h_scales, void* h_out,
               uint8_t* gate_codes, uint8_t* gate_scales, uint8_t* up_codes, uint8_t* up_scales, void* stream)
{
    MXQ_TRY(check_shape(rows, cols, dtype));
    if (half_given(h_codes, h_scales) || half_given(gate_codes, gate_scales) || half_given(up_codes, up_scales) ||
        half_given(gate_codes, up_codes))
        return MXQ_ERR_INVALID_ARG;
    if (cols >= ((int64_t)1 << 30)) return MXQ_ERR_UNSUPPORTED;               // 32-bit places in a row
    if (rows * cols == 0) return MXQ_OK;
    if (!gate || !up || !(h_codes || h_out || gate_codes)) return MXQ_ERR_INVALID_ARG;
    MXQ_TRY(check_rows(gate, ld_gate, rows, cols, dtype));
    MXQ_TRY(check_rows(up, ld_up, rows, cols, dtype));
    if (!aligned(h_codes, 8) || !aligned(h_out, 16) || !aligned(gate_codes, 8) || !aligned(up_codes, 8)) return MXQ_ERR_ALIGNMENT;
    const mxq::SwigluArgs a = {gate, up, ld_gate, ld_up, rows, cols, h_codes, h_scales, h_out, gate_codes, gate_scales, up_codes, up_scales};
    return status(mxq::launch_swiglu(a, dtype, static_cast<hipStream_t>(stream)));
}

int mxq_swiglu_backward(const void* dh, int64_t ld_dh, const uint8_t* gate_codes, const uint8_t* gate_scales,
                        const uint8_t* up_codes, const uint8_t* up_scales, int64_t rows, int64_t cols, int dtype,
                        void* dgate_out, int64_t ld_dgate, void* dup_out, int64_t ld_dup, void* h_out, void* stream)
{
    MXQ_TRY(check_shape(rows, cols, dtype));
    if (cols >= ((int64_t)1 << 30)) return MXQ_ERR_UNSUPPORTED;
    if (rows * cols == 0) return MXQ_OK;
    if (!dh || !gate_codes || !gate_scales || !up_codes || !up_scales || !dgate_out || !dup_out) return MXQ_ERR_INVALID_ARG;
    MXQ_TRY(check_rows(dh, ld_dh, rows, cols, dtype));
    MXQ_TRY(check_rows(dgate_out, ld_dgate, rows, cols, dtype));
    MXQ_TRY(check_rows(dup_out, ld_dup, rows, cols, dtype));
    if (!aligned(gate_codes, 8) || !aligned(up_codes, 8) || !aligned(h_out, 16)) return MXQ_ERR_ALIGNMENT;
    const mxq::SwigluBackArgs a = {dh, gate_codes, gate_scales, up_codes, up_scales, ld_dh, ld_dgate, ld_dup, rows, cols, dgate_out, dup_out, h_out};
    return status(mxq::launch_swiglu_backward(a, dtype, static_cast<hipStream_t>(stream)));
}

size_t mxq_linear_workspace_size(const mxq_linear_args* args)
{
    if (!args || check_linear(*args) != MXQ_OK || args->m == 0 || args->n == 0 || args->k == 0) return 0;
    return mxq::linear_workspace(linear_of(*args));
}

int mxq_linear(const mxq_linear_args* args, void* stream)
{
    if (!args) return MXQ_ERR_INVALID_ARG;
    const mxq_linear_args& g = *args;
    MXQ_TRY(check_linear(g));
    if (!g.tensor_scale_dev && (!(g.tensor_scale > 0.0f) || std::isinf(g.tensor_scale))) return MXQ_ERR_INVALID_ARG;
    if (g.m == 0 || g.n == 0) return MXQ_OK;
    if (!g.y || (g.m > 1 && g.ld_y < g.n)) return MXQ_ERR_INVALID_ARG;
    if (!aligned(g.y, g.y_dtype == MXQ_DT_BF16 ? 2 : 4)) return MXQ_ERR_ALIGNMENT;
    if (g.k > 0) {
        if ((g.x == nullptr) == (g.x_codes == nullptr) || half_given(g.x_codes, g.x_scales)) return MXQ_ERR_INVALID_ARG;
        if (!g.w_codes || !g.w_scales) return MXQ_ERR_INVALID_ARG;
        if (g.x) MXQ_TRY(check_rows(g.x, g.ld_x, g.m, g.k, MXQ_DT_BF16));
        if (!aligned(g.x_codes, 16) || !aligned(g.w_codes, 16) || !aligned(g.w_scales, 4) || !aligned(g.tensor_scale_dev, 4) ||
            !aligned(g.adapter_a, 16) || !aligned(g.adapter_b, 16) || !aligned(g.adapter_scaling, 4) || !aligned(g.adapter_ids, 4))
            return MXQ_ERR_ALIGNMENT;
        const size_t need = mxq_linear_workspace_size(args);
        if (need > 0 && (!g.workspace || g.workspace_bytes < need)) return MXQ_ERR_INVALID_ARG;
        if (need > 0 && !aligned(g.workspace, 16)) return MXQ_ERR_ALIGNMENT;
    }
    return status(mxq::launch_linear(linear_of(g), g.workspace, static_cast<hipStream_t>(stream)));
}

// Which mxq.h and mxq_layers.h this library was built from (for the native calls of the Python binding, which check it).
#ifndef MXQ_HEADER_ID
#define MXQ_HEADER_ID "unknown"
#endif
MXQ_API extern const char mxq_layers_header_id[];
const char mxq_layers_header_id[] = MXQ_HEADER_ID;

}  // extern "C"
