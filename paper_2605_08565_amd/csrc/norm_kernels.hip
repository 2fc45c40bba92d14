// Norm with the residual's addition, and its backward pass from the 8-bit checkpoint (include/mxq_layers.h).
#include "mxq_layers_launch.hpp"
#include "mxq_q8.hpp"

namespace mxq {

namespace {

__device__ __forceinline__ float wave_sum(float v)
{
    v = group_sum<16>(v);
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    return v;
}

// Sum over the threads of a row; every thread gets the same bits.  One row per wavefront (TPR = 64), or one per workgroup.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* slots)
{
    v = wave_sum(v);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63u) == 0u) slots[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) v += slots[i];
    }
    return v;
}

// TPR threads have one row, CH chunks of 8 elements each: thread j has chunks j, TPR + j, ...  The row stays in registers
// between the sum of squares and the outputs, so every input is read once.  Bound by memory: 8192 x 4096 bf16 with residual, dense
// output and checkpoint (303 MB) 54 us, 5.6 TB/s; one row 3.4 us.
template <int DT, int TPR, int CH>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) add_rmsnorm_kernel(NormArgs a)
{
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1;
    __shared__ float slots[16];
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    if (row >= a.rows) return;                              // whole wavefronts; with TPR > 64 whole workgroups
    float t[CH][8];
    float ss = 0.0f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * TPR + lane) * 8;
        if (c < a.cols) {
            load8<DT>(a.x, row * a.ld_x + c, t[k]);
            if (a.residual) {
                float r[8];
                load8<DT>(a.residual, row * a.ld_residual + c, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) t[k][i] += r[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) t[k][i] = 0.0f;
        }
    }
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += t[k][i] * t[k][i];
    ss = row_sum<TPR>(ss, slots);
    // The root in two parts of 32 bits, and the products' low parts with it: an element of 8 bits next to a step's edge falls as its exact value
    // does, but for the last rounding (4096 columns, 153 million elements: 141 a step off, so 88, as with a sum in 64 bits; the time is the same).
    const double r = 1.0 / sqrt((double)ss / a.cols + (double)a.eps);
    const float rstd = (float)r, low = __builtin_isfinite(rstd) ? (float)(r - rstd) : 0.0f;
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * TPR + lane) * 8;
        if (c >= a.cols) continue;
        const int64_t at = row * a.cols + c;
        if (a.hidden) store8<DT>(a.hidden, at, t[k]);
        float y[8], rest[8];                                // y + rest = t * (rstd + low); rest is left out where y is not finite
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = t[k][i] * rstd;
            y[i] = __builtin_isfinite(p) ? __builtin_fmaf(t[k][i], rstd, t[k][i] * low) : p;
            rest[i] = __builtin_fmaf(t[k][i], low, __builtin_fmaf(t[k][i], rstd, -y[i]));
        }
        if (a.n_codes) q8_store(a.n_codes, a.n_scales, at, y);
        if (a.weight) {
            float w[8];
            load8<DT>(a.weight, c, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p = y[i] * w[i];
                y[i] = __builtin_isfinite(p) ? __builtin_fmaf(y[i], w[i], rest[i] * w[i]) : p;
            }
        }
        if (a.y_codes) q8_store(a.y_codes, a.y_scales, at, y);
        if (a.y) store8<DT>(a.y, at, y);
    }
}

// 8 elements as they are in memory.
template <int DT>
struct Raw8 {
    uint4 v[DT == kBF16 ? 1 : 2];
    __device__ void load(const void* p, int64_t first)
    {
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const char*>(p) + first * (DT == kBF16 ? 2 : 4));
        v[0] = q[0];
        if constexpr (DT != kBF16) v[1] = q[1];
    }
    // What was made of it has to be made again.
    __device__ void forget()
    {
        asm volatile("" : "+v"(v[0].x), "+v"(v[0].y), "+v"(v[0].z), "+v"(v[0].w));
        if constexpr (DT != kBF16) asm volatile("" : "+v"(v[1].x), "+v"(v[1].y), "+v"(v[1].z), "+v"(v[1].w));
    }
    __device__ void widen(float (&f)[8]) const
    {
        const uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == kBF16) {
                f[2 * i] = u2f(w[i] << 16);
                f[2 * i + 1] = u2f(w[i] & 0xFFFF0000u);
            } else {
                const uint32_t h[4] = {v[1].x, v[1].y, v[1].z, v[1].w};
                f[i] = u2f(w[i]);
                f[4 + i] = u2f(h[i]);
            }
        }
    }
};

// A group of TPR threads goes over rows g, g + groups, ... and keeps its part of the weight's gradient in registers; what is
// left at the end is one row of partial sums per group, added up by norm_weight_kernel in the groups' order.  Bound by memory: the
// next row is loaded, as it is, while this one is summed (behind its last one a group loads that one again, for nothing: never a row
// that another group may be writing, where dx is dy or dhidden itself).  8192 x 4096 bf16 with dhidden (236 MB and 8 MB of partial sums)
// 78 -> 41 us by that, 5.9 TB/s; 512 groups against 256, 384, 768 and 1024: 44.8 us with the second launch, 51.1, 52.8, 48.2, 52.4.
//
// Rows of 1024 threads are tight: a thread has 128 registers, and two rows with the weight and its gradient do not fit (they spilled
// 25 registers in bf16 and 101 in fp32).  There the weight and its gradient are in LDS, a place for each thread, dhidden is loaded with
// its row and not ahead of it, and what was widened for the sum is widened once more for dx.  With the second launch, 2048 x 16384 with
// dhidden 120 -> 66 us in bf16 and 321 -> 119 in fp32, 2048 x 8224 74 -> 37 and 147 -> 46.
template <int DT, int TPR, int CH>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) add_rmsnorm_backward_kernel(NormBackArgs a, int64_t groups)
{
    constexpr int kRows = TPR < 256 ? 256 / TPR : 1;
    constexpr bool kTight = TPR == 1024;
    __shared__ float slots[2][16];
    __shared__ Raw8<DT> weights[kTight ? CH : 1][kTight ? TPR : 1];        // tight: a thread's part of the weight, and of its gradient
    __shared__ f32x4 dw_parts[kTight ? 2 * CH : 1][kTight ? TPR : 1];
    const int lane = threadIdx.x % TPR;
    const int64_t group = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    if (group >= groups) return;
    struct Row {
        Raw8<DT> dy[CH], dh[kTight ? 1 : CH];
        uint2 n[CH];
        uint32_t scale[CH];
        float rstd;
    };
    auto load = [&](int64_t row, Row& r) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * TPR + lane) * 8;
            if (c < a.cols) {
                const int64_t at = row * a.cols + c;
                r.dy[k].load(a.dy, row * a.ld_dy + c);
                r.n[k] = *reinterpret_cast<const uint2*>(a.n_codes + at);
                r.scale[k] = a.n_scales[at >> 5];
                if constexpr (!kTight)
                    if (a.dhidden) r.dh[k].load(a.dhidden, row * a.ld_dhidden + c);
            }
        }
        r.rstd = a.rstd[row];
    };
    Raw8<DT> weight[kTight ? 1 : CH];
#pragma unroll
    for (int k = 0; k < CH; ++k)
        if (a.weight && (k * TPR + lane) * 8 < a.cols) {
            if constexpr (kTight) weights[k][lane].load(a.weight, (k * TPR + lane) * 8);
            else weight[k].load(a.weight, (k * TPR + lane) * 8);
        }
    float dw[CH][8] = {};
    if constexpr (kTight) {
#pragma unroll
        for (int j = 0; j < 2 * CH; ++j) dw_parts[j][lane] = f32x4{};
    }
    int parity = 0;
    Row now = {}, next = {};
    load(group, now);
    for (int64_t row = group; row < a.rows; row += groups, parity ^= 1) {
        Raw8<DT> dh[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if constexpr (!kTight) dh[k] = now.dh[k];
            else if (a.dhidden && (k * TPR + lane) * 8 < a.cols) dh[k].load(a.dhidden, row * a.ld_dhidden + (k * TPR + lane) * 8);
        }
        load(row + groups < a.rows ? row + groups : row, next);
        // dy and n of a chunk, zeros behind the row's end; and g in the place of dy.
        auto widen = [&](int k, float (&d)[8], float (&n)[8]) {
            const bool in = (k * TPR + lane) * 8 < a.cols;
            now.dy[k].widen(d);
            q8_widen(now.n[k], q8_scale(now.scale[k]), n);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!in) d[i] = n[i] = 0.0f;
        };
        auto weigh = [&](int k, float (&d)[8]) {
            if (!a.weight) return;
            const bool in = (k * TPR + lane) * 8 < a.cols;
            float w[8];
            if constexpr (kTight) weights[k][lane].widen(w);
            else weight[k].widen(w);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = in ? d[i] * w[i] : 0.0f;
        };
        float g[kTight ? 1 : CH][8], n[kTight ? 1 : CH][8];
        float along = 0.0f;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int at = kTight ? 0 : k;
            widen(k, g[at], n[at]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (kTight) dw_parts[2 * k + i / 4][lane][i % 4] += g[at][i] * n[at][i];
                else dw[k][i] += g[at][i] * n[at][i];
            }
            weigh(k, g[at]);
#pragma unroll
            for (int i = 0; i < 8; ++i) along += g[at][i] * n[at][i];
        }
        along = row_sum<TPR>(along, slots[parity]) / (float)a.cols;       // the other slots may still be read: two in turn
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = (k * TPR + lane) * 8, at = kTight ? 0 : k;
            if (c >= a.cols) continue;
            if constexpr (kTight) {
                now.dy[k].forget();                         // or the compiler keeps what was widened
                asm volatile("" : "+v"(now.n[k].x), "+v"(now.n[k].y));
                widen(k, g[0], n[0]);
                weigh(k, g[0]);
            }
            float dx[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) dx[i] = now.rstd * (g[at][i] - n[at][i] * along);
            if (a.dhidden) {
                float d[8];
                dh[k].widen(d);
#pragma unroll
                for (int i = 0; i < 8; ++i) dx[i] += d[i];
            }
            store8<DT>(a.dx, row * a.cols + c, dx);
        }
        now = next;
    }
    if (!a.dweight) return;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = (k * TPR + lane) * 8;
        if constexpr (kTight) {
#pragma unroll
            for (int i = 0; i < 8; ++i) dw[k][i] = dw_parts[2 * k + i / 4][lane][i % 4];
        }
        if (c < a.cols) store8<kF32>(a.partial, group * a.cols + c, dw[k]);
    }
}

// dweight[c] = sum over groups of partial[group][c]: 32 columns a workgroup, 8 threads for a row of them, 128 rows at a time.  Bound by
// its launch and one trip to memory (512 groups of 4096: 8 MB).
__global__ void __launch_bounds__(1024) norm_weight_kernel(const float* __restrict__ partial, int64_t groups, int cols, float* __restrict__ out)
{
    __shared__ f32x4 sums[128][8];
    const int j = threadIdx.x & 7, s = threadIdx.x >> 3, c = blockIdx.x * 32 + 4 * j;     // cols is a multiple of 32
    f32x4 v = {};
#pragma unroll 4
    for (int64_t g = s; g < groups; g += 128) v += *reinterpret_cast<const f32x4*>(partial + g * cols + c);
    sums[s][j] = v;
    __syncthreads();
    if (s >= 8) return;                                                                  // the first wavefront
#pragma unroll
    for (int i = 1; i < 16; ++i) v += sums[s + 8 * i][j];
#pragma unroll
    for (int d = 8; d < 64; d *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += __shfl_xor(v[i], d);
    if (s == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) out[c + i] = v[i];                                   // aligned to its elements only
}

// Threads to a row and chunks to a thread.
struct Shape { int tpr, ch; };

Shape shape_of(int64_t cols)
{
    const int64_t chunks = cols / 8;
    const int tpr = chunks <= 128 ? 64 : chunks <= 1024 ? 256 : 1024;
    return {tpr, (int)((chunks + tpr - 1) / tpr)};
}

template <int N>
using Int = std::integral_constant<int, N>;

template <class F>
void by_shape(Shape s, F f)
{
    switch (s.tpr * 16 + s.ch) {
        case 64 * 16 + 0:                                                                    // no columns: not called
        case 64 * 16 + 1: f(Int<64>(), Int<1>()); break;
        case 64 * 16 + 2: f(Int<64>(), Int<2>()); break;
        case 256 * 16 + 1: f(Int<256>(), Int<1>()); break;
        case 256 * 16 + 2: f(Int<256>(), Int<2>()); break;
        case 256 * 16 + 3: f(Int<256>(), Int<3>()); break;
        case 256 * 16 + 4: f(Int<256>(), Int<4>()); break;
        default: f(Int<1024>(), Int<2>()); break;                                            // 16384 columns
    }
}

template <int DT>
void launch_norm(const NormArgs& a, hipStream_t stream)
{
    by_shape(shape_of(a.cols), [&](auto tpr, auto ch) {
        constexpr int kThreadsHere = tpr < 256 ? 256 : tpr, kRows = kThreadsHere / tpr;
        hipLaunchKernelGGL((add_rmsnorm_kernel<DT, tpr, ch>), dim3((unsigned)((a.rows + kRows - 1) / kRows)), dim3(kThreadsHere), 0, stream, a);
    });
}

template <int DT>
void launch_norm_back(const NormBackArgs& a, hipStream_t stream)
{
    const int64_t groups = norm_back_groups(a.rows, a.cols);
    by_shape(shape_of(a.cols), [&](auto tpr, auto ch) {
        constexpr int kThreadsHere = tpr < 256 ? 256 : tpr, kRows = kThreadsHere / tpr;
        hipLaunchKernelGGL((add_rmsnorm_backward_kernel<DT, tpr, ch>), dim3((unsigned)((groups + kRows - 1) / kRows)), dim3(kThreadsHere), 0,
                           stream, a, groups);
    });
}

}  // namespace

int64_t norm_back_groups(int64_t rows, int64_t cols)
{
    int64_t most = cols > 0 ? (1 << 21) / cols : 1;               // 8 MiB of partial sums, measured at 4096 columns (above) and there alone
    most = most < 64 ? 64 : most > 4096 ? 4096 : most;
    return rows < most ? rows : most;
}

hipError_t launch_add_rmsnorm(const NormArgs& a, int dtype, hipStream_t stream)
{
    // a launch's grid counts 32-bit work items: rows in pieces
    constexpr int64_t kPiece = 1 << 20;
    const int64_t size = dtype == kBF16 ? 2 : 4;
    for (int64_t r = 0; r < a.rows; r += kPiece) {
        NormArgs p = a;
        const int64_t at = r * a.cols;
        p.rows = a.rows - r < kPiece ? a.rows - r : kPiece;
        p.x = (const char*)a.x + r * a.ld_x * size;
        if (a.residual) p.residual = (const char*)a.residual + r * a.ld_residual * size;
        if (a.hidden) p.hidden = (char*)a.hidden + at * size;
        if (a.y) p.y = (char*)a.y + at * size;
        if (a.y_codes) { p.y_codes += at; p.y_scales += at / 32; }
        if (a.n_codes) { p.n_codes += at; p.n_scales += at / 32; }
        if (a.rstd) p.rstd += r;
        if (dtype == kBF16) launch_norm<kBF16>(p, stream);
        else launch_norm<kF32>(p, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_add_rmsnorm_backward(const NormBackArgs& a, int dtype, hipStream_t stream)
{
    const int64_t groups = norm_back_groups(a.rows, a.cols);
    if (groups > 0) {
        if (dtype == kBF16) launch_norm_back<kBF16>(a, stream);
        else launch_norm_back<kF32>(a, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.dweight)
        hipLaunchKernelGGL(norm_weight_kernel, dim3((unsigned)(a.cols / 32)), dim3(1024), 0, stream, a.partial, groups, a.cols, a.dweight);
    return hipGetLastError();
}

}  // namespace mxq
