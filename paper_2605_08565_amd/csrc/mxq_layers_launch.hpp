// Host-side launch descriptors of the layer operators, after validation.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mxq {

struct NormArgs {
    const void* x;
    const void* residual;      // or NULL
    const void* weight;        // or NULL
    int64_t ld_x, ld_residual, rows;
    int cols;
    float eps;
    void* hidden;              // or NULL
    uint8_t* y_codes;          // or NULL
    uint8_t* y_scales;
    void* y;                   // or NULL
    uint8_t* n_codes;          // or NULL
    uint8_t* n_scales;
    float* rstd;               // or NULL
};

struct NormBackArgs {
    const void* dy;
    const uint8_t* n_codes;
    const uint8_t* n_scales;
    const float* rstd;
    const void* weight;        // or NULL
    const void* dhidden;       // or NULL
    int64_t ld_dy, ld_dhidden, rows;
    int cols;
    void* dx;
    float* dweight;            // or NULL
    float* partial;            // norm_back_groups() rows of cols sums
};

struct SwigluArgs {
    const void* gate;
    const void* up;
    int64_t ld_gate, ld_up, rows, cols;
    uint8_t* h_codes;          // or NULL
    uint8_t* h_scales;
    void* h;                   // or NULL
    uint8_t* gate_codes;       // or NULL
    uint8_t* gate_scales;
    uint8_t* up_codes;
    uint8_t* up_scales;
};

struct SwigluBackArgs {
    const void* dh;
    const uint8_t* gate_codes;
    const uint8_t* gate_scales;
    const uint8_t* up_codes;
    const uint8_t* up_scales;
    int64_t ld_dh, ld_dgate, ld_dup, rows, cols;
    void* dgate;
    void* dup;
    void* h;                   // or NULL
};

struct LinearArgs {
    const void* x;             // bf16, or NULL
    int64_t ld_x;
    const uint8_t* x_codes;    // Q8, or NULL
    const uint8_t* x_scales;
    int m, n, k;
    const uint8_t* w_codes;
    const uint8_t* w_scales;
    int block, scale_fmt;
    float T;
    const float* t_dev;        // or NULL
    const uint16_t* a;         // or NULL: no adapters
    const uint16_t* b;
    const float* scaling;
    const int32_t* ids;        // or NULL: adapter 0
    int count, rank;
    void* y;
    int64_t ld_y;
    int y_dtype;
    bool mx_sums;              // the scaled instruction's sums will do
    // set by the launch
    float* low;                // low_parts x m x rank: scaling * x * A^T, in parts of k to be added up
    int low_parts, low_slots;  // low_slots: different adapters that 16 rows can have
    int low_blocks;            // workgroups of the direct kernel that form `low`
    float* parts;              // splits x tiles of 16 x 16: sums over parts of k; NULL if a workgroup has all of k
    int splits, chunks_each;   // parts of k, and their length in chunks of 128
};

// Rows of partial sums that the backward pass of the norm leaves: its workgroups' number of row groups.
int64_t norm_back_groups(int64_t rows, int64_t cols);

hipError_t launch_add_rmsnorm(const NormArgs& a, int dtype, hipStream_t stream);
hipError_t launch_add_rmsnorm_backward(const NormBackArgs& a, int dtype, hipStream_t stream);
hipError_t launch_swiglu(const SwigluArgs& a, int dtype, hipStream_t stream);
hipError_t launch_swiglu_backward(const SwigluBackArgs& a, int dtype, hipStream_t stream);

size_t linear_workspace(const LinearArgs& a);
hipError_t launch_linear(const LinearArgs& a, void* workspace, hipStream_t stream);

}  // namespace mxq
