// Gated activation between two projections and its backward pass from the 8-bit checkpoint (include/mxq_layers.h).
#include "mxq_layers_launch.hpp"
#include "mxq_q8.hpp"

namespace mxq {

namespace {

__device__ __forceinline__ float sigmoid(float g) { return 1.0f / (1.0f + expf(-g)); }

// Row and column of a thread's chunk of 8 elements: the workgroup's first chunk divided on the scalar unit, the lanes in 32 bits.
struct Place {
    int64_t row;
    uint32_t col;
    bool in;
    __device__ Place(int64_t rows, int64_t cols)
    {
        const uint64_t per_row = (uint64_t)cols / 8, first = (uint64_t)blockIdx.x * kThreadsHere;
        const uint64_t row0 = first / per_row;
        const uint32_t rest = (uint32_t)(first - row0 * per_row) + threadIdx.x, down = rest / (uint32_t)per_row;
        row = (int64_t)row0 + down;
        col = (rest - down * (uint32_t)per_row) * 8u;
        in = row < rows;
    }
    static constexpr int kThreadsHere = 256;
};

// One lane has 8 consecutive elements; blocks of 32 are quads of lanes, and all of a quad is inside or none.  No loop and no LDS: bound
// by memory.  4096 x 14336 bf16, dense output and checkpoint (473 MB) 87 us, 5.4 TB/s; 16 rows 2.8 us.
template <int DT>
__global__ void __launch_bounds__(256) swiglu_kernel(SwigluArgs a)
{
    const Place p(a.rows, a.cols);
    if (!p.in) return;
    float g[8], u[8], h[8];
    load8<DT>(a.gate, p.row * a.ld_gate + p.col, g);
    load8<DT>(a.up, p.row * a.ld_up + p.col, u);
    const int64_t at = p.row * a.cols + p.col;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = g[i] * sigmoid(g[i]) * u[i];
    if (a.h_codes) q8_store(a.h_codes, a.h_scales, at, h);
    if (a.h) store8<DT>(a.h, at, h);
    if (a.gate_codes) {
        q8_store(a.gate_codes, a.gate_scales, at, g);
        q8_store(a.up_codes, a.up_scales, at, u);
    }
}

// 4096 x 14336 bf16 with the output again (591 MB) 111 to 115 us, 5.2 TB/s.
template <int DT>
__global__ void __launch_bounds__(256) swiglu_backward_kernel(SwigluBackArgs a)
{
    const Place p(a.rows, a.cols);
    if (!p.in) return;
    const int64_t at = p.row * a.cols + p.col;
    float g[8], u[8], d[8], dg[8], du[8], h[8];
    load8<DT>(a.dh, p.row * a.ld_dh + p.col, d);
    q8_widen(*reinterpret_cast<const uint2*>(a.gate_codes + at), q8_scale(a.gate_scales[at >> 5]), g);
    q8_widen(*reinterpret_cast<const uint2*>(a.up_codes + at), q8_scale(a.up_scales[at >> 5]), u);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float s = sigmoid(g[i]), act = g[i] * s;
        dg[i] = d[i] * u[i] * (s * (1.0f + g[i] * (1.0f - s)));
        du[i] = d[i] * act;
        h[i] = act * u[i];
    }
    store8<DT>(a.dgate, p.row * a.ld_dgate + p.col, dg);
    store8<DT>(a.dup, p.row * a.ld_dup + p.col, du);
    if (a.h) store8<DT>(a.h, at, h);
}

// Workgroups that cover `rows` rows, and how many rows a launch may have (its grid counts 32-bit work items).
unsigned tiles(int64_t rows, int64_t cols) { return (unsigned)((rows * (cols / 8) + Place::kThreadsHere - 1) / Place::kThreadsHere); }

int64_t rows_a_launch(int64_t cols)
{
    const int64_t r = ((int64_t)1 << 30) / (cols / 8);
    return r < 1 ? 1 : r;
}

}  // namespace

hipError_t launch_swiglu(const SwigluArgs& a, int dtype, hipStream_t stream)
{
    const int64_t size = dtype == kBF16 ? 2 : 4, piece = rows_a_launch(a.cols);
    for (int64_t r = 0; r < a.rows; r += piece) {
        SwigluArgs p = a;
        const int64_t at = r * a.cols;
        p.rows = a.rows - r < piece ? a.rows - r : piece;
        p.gate = (const char*)a.gate + r * a.ld_gate * size;
        p.up = (const char*)a.up + r * a.ld_up * size;
        if (a.h_codes) { p.h_codes += at; p.h_scales += at / 32; }
        if (a.h) p.h = (char*)a.h + at * size;
        if (a.gate_codes) { p.gate_codes += at; p.gate_scales += at / 32; p.up_codes += at; p.up_scales += at / 32; }
        if (dtype == kBF16) hipLaunchKernelGGL(swiglu_kernel<kBF16>, dim3(tiles(p.rows, p.cols)), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL(swiglu_kernel<kF32>, dim3(tiles(p.rows, p.cols)), dim3(256), 0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_swiglu_backward(const SwigluBackArgs& a, int dtype, hipStream_t stream)
{
    const int64_t size = dtype == kBF16 ? 2 : 4, piece = rows_a_launch(a.cols);
    for (int64_t r = 0; r < a.rows; r += piece) {
        SwigluBackArgs p = a;
        const int64_t at = r * a.cols;
        p.rows = a.rows - r < piece ? a.rows - r : piece;
        p.dh = (const char*)a.dh + r * a.ld_dh * size;
        p.gate_codes += at; p.gate_scales += at / 32; p.up_codes += at; p.up_scales += at / 32;
        p.dgate = (char*)a.dgate + r * a.ld_dgate * size;
        p.dup = (char*)a.dup + r * a.ld_dup * size;
        if (a.h) p.h = (char*)a.h + at * size;
        if (dtype == kBF16) hipLaunchKernelGGL(swiglu_backward_kernel<kBF16>, dim3(tiles(p.rows, p.cols)), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL(swiglu_backward_kernel<kF32>, dim3(tiles(p.rows, p.cols)), dim3(256), 0, stream, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace mxq
