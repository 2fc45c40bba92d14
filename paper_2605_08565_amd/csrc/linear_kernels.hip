// Projections over packed FP4 weights, with low-rank adapters beside them (include/mxq_layers.h).
#include "linear_plan.hpp"
#include "mxq_layers_launch.hpp"
#include "mxq_q8.hpp"

#include <type_traits>

namespace mxq {

namespace {

using i32x8 = int __attribute__((ext_vector_type(8)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

enum : int { kXBf16 = 0, kXQ8 = 1, kXMx = 2 };       // activations: bf16; Q8 widened to bf16; Q8 as it is (power-of-two scales)

// ---------------------------------------------------------------------------------------
// Fragments.  The weights are the first operand, so a tile of the result has 16 weight rows (columns of y) down and
// 16 tokens across: lane l has token l % 16 and the four columns 4 * (l / 16) .. + 3, consecutive in y.  Each lane loads 32
// consecutive elements of k for its row: group g = l / 16 has k0 + 32 g .. + 31 of a chunk of 128.  The order of k within a
// contraction is free as long as both operands have the same, so four products of 32 take 8 elements each from every group.
// ---------------------------------------------------------------------------------------

// 8 codes (one dword) times their scale, as bf16: at most 2 + 4 significant bits, exact.
__device__ __forceinline__ uint4 widen_codes(uint32_t c, float S)
{
    float q[8];
    e2m1_unpack8(c, 1.0f, q);
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] *= S;
    return bf16_of8(q);
}

__device__ __forceinline__ f32x4 mfma_bf16(uint4 a, uint4 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Scale bytes of any format without branches.  E4M3 and UE5M3 read as the top bits of an fp32 number are off by the difference of the
// biases alone, sub-normals included: one product.  E8M0 is the exponent itself; its byte 0 (2^-127) is a sub-normal fp32 number.
struct ScaleReader {
    int shift;
    uint32_t least, most;
    float mul;
    __device__ explicit ScaleReader(int fmt)
        : shift(fmt == kE8M0 ? 23 : 20), least(fmt == kE8M0 ? 0x00400000u : 0u),
          most(fmt == kE8M0 ? 254u : fmt == kE4M3 ? (uint32_t)ScaleFmt<kE4M3>::kMaxCode : (uint32_t)ScaleFmt<kUE5M3>::kMaxCode),
          mul(fmt == kE8M0 ? 1.0f : u2f((uint32_t)(254 - (fmt == kE4M3 ? ScaleFmt<kE4M3>::kBias : ScaleFmt<kUE5M3>::kBias)) << 23)) {}
    __device__ __forceinline__ float operator()(uint32_t code) const
    {
        const float v = u2f(max(code << shift, least)) * mul;
        return code > most ? u2f(0x7FC00000u) : v;
    }
};

// Loads through a buffer descriptor: scalar base, 32-bit offset of the lane, scalar offset; beyond the end they give zeros.  (With
// pointers the compiler keeps a 64-bit address a lane for every load of a loop, more registers than the tiles below leave.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}
constexpr uint32_t kNowhere = 0xFFFFFFF0u;            // an offset beyond every buffer
__device__ __forceinline__ uint4 buffer_load16(__amdgpu_buffer_rsrc_t b, uint32_t at, int scalar)
{
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(b, (int)at, scalar, 0));
}
// Four scale bytes (SB = 8: those of 32 elements), or one in the low byte.
template <int SB>
__device__ __forceinline__ uint32_t buffer_load_scales(__amdgpu_buffer_rsrc_t b, uint32_t at, int scalar)
{
    if constexpr (SB == 8) return __builtin_amdgcn_raw_buffer_load_b32(b, (int)at, scalar, 0);
    else return (uint8_t)__builtin_amdgcn_raw_buffer_load_b8(b, (int)at, scalar, 0);
}

// Adapter of a token, -1 for none.
__device__ __forceinline__ int adapter_of(const LinearArgs& a, int m)
{
    if (m >= a.m) return -1;
    const int id = a.ids ? a.ids[m] : 0;
    return (unsigned)id < (unsigned)a.count ? id : -1;
}

__device__ __forceinline__ void store_y(const LinearArgs& a, int m, int n, f32x4 v)
{
    if (m >= a.m || n >= a.n) return;
    const int64_t at = (int64_t)m * a.ld_y + n;
    if (a.y_dtype == kBF16) {
        uint16_t* p = static_cast<uint16_t*>(a.y) + at;
        const uint32_t lo = bf16_pair(v[0], v[1]), hi = bf16_pair(v[2], v[3]);
        if (n + 4 <= a.n && (reinterpret_cast<uintptr_t>(p) & 7u) == 0u) {
            *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < a.n) p[i] = (uint16_t)((i < 2 ? lo : hi) >> (16 * (i & 1)));
        }
    } else {
        float* p = static_cast<float*>(a.y) + at;
        if (n + 4 <= a.n && (reinterpret_cast<uintptr_t>(p) & 15u) == 0u) {
            *reinterpret_cast<f32x4*>(p) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < a.n) p[i] = v[i];
        }
    }
}

// The top halves of 8 values: bf16 that is cut off.
__device__ __forceinline__ uint4 cut_of8(const float (&v)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f2u(v[2 * i]) >> 16 | (f2u(v[2 * i + 1]) & 0xFFFF0000u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 8 bf16 values with zeros in place of infinities and NaN.
__device__ __forceinline__ uint4 finite_of8(uint4 v)
{
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x00007F80u) == 0x00007F80u) w[i] &= 0xFFFF0000u;
        if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0x0000FFFFu;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Adds B_a * low^T to NT tiles, side by side, of the same 16 tokens: one adapter after the other, each kept by its tokens alone (not
// added as zeros to the others, where an infinity in B would be NaN).  `low` (fp32) enters as three bf16 parts of 8 bits, cut off and
// not rounded: all of its 24 bits, and none of them beyond bf16's range.  Infinities of `low` and of B meet the first part alone, which has
// the sign of the whole: the others would be infinity - infinity, or 0 * infinity.
template <int NT>
__device__ __forceinline__ void add_adapters(const LinearArgs& a, int m, int n0, f32x4 (&acc)[NT])
{
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int id = adapter_of(a, m);
    uint64_t left = __builtin_amdgcn_ballot_w64(id >= 0);
    while (left != 0ull) {
        const int cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        const bool mine = id == cur;
        f32x4 sum[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) sum[i] = acc[i];
        for (int r0 = 0; r0 < a.rank; r0 += 32) {
            const int r = r0 + 8 * g;
            float u[8] = {}, mid[8], rest[8];
            if (r < a.rank && mine) {
                load8<kF32>(a.low, (int64_t)m * a.rank + r, u);
                for (int p = 1; p < a.low_parts; ++p) {
                    float more[8];
                    load8<kF32>(a.low, ((int64_t)p * a.m + m) * a.rank + r, more);
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] += more[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                mid[i] = __builtin_isfinite(u[i]) ? u[i] - u2f(f2u(u[i]) & 0xFFFF0000u) : 0.0f;
                rest[i] = mid[i] - u2f(f2u(mid[i]) & 0xFFFF0000u);
            }
            const uint4 first = cut_of8(u), second = cut_of8(mid), third = cut_of8(rest);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                uint4 w = make_uint4(0u, 0u, 0u, 0u);
                if (r < a.rank) w = *reinterpret_cast<const uint4*>(a.b + ((int64_t)cur * a.n + min(n0 + 16 * i + (lane & 15), a.n - 1)) * a.rank + r);
                const uint4 finite = finite_of8(w);
                sum[i] = mfma_bf16(finite, third, sum[i]);             // the small ones first
                sum[i] = mfma_bf16(finite, second, sum[i]);
                sum[i] = mfma_bf16(w, first, sum[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[i] = mine ? sum[i] : acc[i];
        left &= ~__builtin_amdgcn_ballot_w64(mine);
    }
}

// 8 elements of a row of activations as bf16.
template <int XT>
__device__ __forceinline__ uint4 load_x8(const LinearArgs& a, int m, int k)
{
    if constexpr (XT == kXBf16) {
        return *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.x) + (int64_t)m * a.ld_x + k);
    } else {
        const int64_t at = (int64_t)m * a.k + k;
        float v[8];
        q8_widen(*reinterpret_cast<const uint2*>(a.x_codes + at), q8_scale(a.x_scales[at >> 5]), v);
        return bf16_of8(v);
    }
}

// Sums over a part of k leave a workgroup as whole tiles of 16 x 16 in the order of their registers: 1 KiB that a wavefront
// writes and reads in one piece.
__device__ __forceinline__ f32x4* part_tile(const LinearArgs& a, int split, int m, int n)
{
    const int64_t mt = (a.m + 15) / 16, nt = (a.n + 15) / 16;
    return reinterpret_cast<f32x4*>(a.parts) + (((int64_t)split * mt + m / 16) * nt + n / 16) * 64;
}

// ---------------------------------------------------------------------------------------
// Adapters, first product: low[m, r] = scaling * sum_k x[m, k] A[r, k].  A workgroup has 16 tokens, 16 rows of A, the slot-th
// of the tokens' different adapters (in the order of their first tokens) and one part of k, which its wavefronts take in turn.
// ---------------------------------------------------------------------------------------
constexpr int kWaves = kLinearWaves;

template <int XT>
__device__ __forceinline__ void lowrank_block(const LinearArgs& a, int block, f32x4 (&sums)[kWaves][64])
{
    constexpr int kAhead = 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int rt = (a.rank + 15) / 16;
    // Slots last: those beyond a tile's adapters are empty, and every eighth, say, workgroup with work would lie on every eighth unit
    // (2048 tokens sorted by their 8 adapters, k = 14336: 98 us, one adapter 10).
    const int mt = (a.m + 15) / 16;
    const int part = block % a.low_parts, r0 = block / a.low_parts % rt * 16, slot = block / (a.low_parts * rt * mt);
    const int m = block / (a.low_parts * rt) % mt * 16 + (lane & 15);
    const int id = adapter_of(a, m);
    uint64_t left = __builtin_amdgcn_ballot_w64(id >= 0);
    int cur = -1;
    for (int i = 0; i <= slot; ++i) {
        if (left == 0ull) return;                      // the same in every wavefront
        cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        left &= ~__builtin_amdgcn_ballot_w64(id == cur);
    }
    const int row = min(m, a.m - 1);
    const uint16_t* w = a.a + ((int64_t)cur * a.rank + min(r0 + (lane & 15), a.rank - 1)) * a.k + 8 * g;
    const int steps = a.k / 32, each = (steps + a.low_parts - 1) / a.low_parts, end = min(steps, (part + 1) * each);
    f32x4 acc = {};
    for (int s = part * each + wave; s < end; s += kWaves * kAhead) {
        uint4 av[kAhead] = {}, xv[kAhead] = {};
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (s + i * kWaves < end) {
                av[i] = *reinterpret_cast<const uint4*>(w + (s + i * kWaves) * 32);
                xv[i] = load_x8<XT>(a, row, (s + i * kWaves) * 32 + 8 * g);
            }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) acc = mfma_bf16(av[i], xv[i], acc);
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave != 0 || id != cur) return;
    f32x4 v = sums[0][lane];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) v += sums[i][lane];
    const int r = r0 + 4 * g;
    if (r < a.rank) *reinterpret_cast<f32x4*>(a.low + ((int64_t)part * a.m + m) * a.rank + r) = v * a.scaling[cur];
}

template <int XT>
__global__ void __launch_bounds__(64 * kWaves) lowrank_kernel(LinearArgs a)
{
    __shared__ f32x4 sums[kWaves][64];
    lowrank_block<XT>(a, blockIdx.x, sums);
}

// 16 bytes a lane from a buffer to LDS, lane l to `lds` + 16 l, no registers in between; zeros for an offset beyond the buffer.  Not
// counted by the compiler: the caller waits with all_loads_done().  m0, which holds the place in LDS, is an operand: the compiler writes it
// and knows that it has (one wait state has to lie between that and the load).
using i32x4 = int __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void load_to_lds(i32x4 buffer, uint32_t at, int scalar, uint32_t lds)
{
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"{m0}"(lds), "v"(at), "s"(buffer), "s"(scalar) : "memory");
}
// The four words of a descriptor as buffer_of() makes it: address, no stride, size, format.
__device__ __forceinline__ i32x4 buffer_words(const void* base, uint32_t bytes)
{
    const uint64_t p = reinterpret_cast<uint64_t>(base);
    return {__builtin_amdgcn_readfirstlane((int)(uint32_t)p), __builtin_amdgcn_readfirstlane((int)(p >> 32)),
            __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
}
// All but the last N.
template <int N>
__device__ __forceinline__ void loads_done_but()
{
    static_assert(N < 64, "six bits");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
    asm volatile("" ::: "memory");
}
__device__ __forceinline__ uint32_t lds_of(const void* p) { return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)p); }
// s_waitcnt vmcnt(0).  The builtin, which the compiler sees: behind it, it does not wait for registers loaded before.
__device__ __forceinline__ void all_loads_done()
{
    __builtin_amdgcn_s_waitcnt(0x0F70);
    asm volatile("" ::: "memory");
}

template <int XT>
__device__ __forceinline__ uint32_t piece_of(uint32_t row, uint32_t piece)
{
    return XT == kXMx ? piece ^ (row & 7u) : piece ^ (row & 15u);
}

// ---------------------------------------------------------------------------------------
// Few tokens: the weights straight from memory to the registers of the wavefront that multiplies them, everything else through LDS.  A
// workgroup has NT * 16 rows of W, all tokens (MT * 16) and one part of k, whose chunks of 128 its eight wavefronts take in turn;
// they join their sums in LDS.  The last workgroups of the launch form the adapters' first product meanwhile, and
// linear_join_few_kernel behind it adds what depends on both.
//
// What bounds it: the bytes of W.  Reading 14336 x 2048 bytes of codes 16 rows at a time takes 6.2 us and is as fast as reading them
// in a line (5.9).  A lane needs 1 to 4 scale bytes of each row for a chunk: loaded by the lanes that need them they cost 3.5 us of 12.1
// (7 of 20.2 with 28672 rows), because every such load touches 16 lines for a few bytes of each; they come to LDS in whole lines
// instead, once a workgroup, and so do the activations, which every wavefront would load again.  One token, 14336 x 4096 E4M3 (33 MB)
// 10.7 us; Q8 against E8M0, one token, 28672 x 4096 (62 MB) 23.1 us, by the scaled instruction 15.7; 24 tokens x 4096 x 14336 15.1 and
// 11.3.  The widening, two instructions a weight, is 3.9 us of the first if nothing hides it: small workgroups, so that some load while
// others multiply.
// ---------------------------------------------------------------------------------------
template <int XT, int SB, int NT, int MT, int AHEAD>
__global__ void __launch_bounds__(64 * kWaves) linear_direct_kernel(LinearArgs a, int main_blocks, DirectLds lds)
{
    constexpr int kRow = XT == kXBf16 ? 256 : 128;     // bytes of a chunk of one token
    extern __shared__ __align__(16) uint8_t xs[];      // tokens (later the sums), scales of tokens, scales of W
    uint32_t* x_scales = reinterpret_cast<uint32_t*>(xs + lds.x_scales);               // four bytes for the 128 of a chunk
    uint32_t* w_scales = reinterpret_cast<uint32_t*>(xs + lds.w_scales);
    if ((int)blockIdx.x >= main_blocks) {
        if (blockIdx.z == 0) lowrank_block<XT == kXMx ? (int)kXQ8 : XT>(a, blockIdx.x - main_blocks, *reinterpret_cast<f32x4(*)[kWaves][64]>(xs));
        return;
    }
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r16 = lane & 15;
    const int n0 = (int)blockIdx.x * (16 * NT);
    const int shift = __builtin_ctz(a.block), per_row = a.k >> shift;
    const int n_last = min(a.n - 1 - n0, NT * 16 - 1), m_last = a.m - 1;
    const int first = blockIdx.z * a.chunks_each, end = min((a.k + 127) / 128, first + a.chunks_each);
    const __amdgpu_buffer_rsrc_t codes = buffer_of(a.w_codes + (int64_t)n0 * (a.k / 2), (uint32_t)(n_last + 1) * (uint32_t)(a.k / 2));
    uint32_t code_at[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) code_at[i] = (uint32_t)min(16 * i + r16, n_last) * (uint32_t)(a.k / 2) + 16u * g;
    struct Group {                                     // of AHEAD chunks
        uint4 c[AHEAD][NT];
    };
    auto load = [&](int c0, Group& f) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int chunk = c0 + u * kWaves;
            const bool in = chunk < end && chunk * 128 + 32 * g < a.k;       // k is a multiple of 32: all of a lane's 32 or none
#pragma unroll
            for (int i = 0; i < NT; ++i) f.c[u][i] = buffer_load16(codes, in ? code_at[i] : kNowhere, chunk * 64);
        }
        __builtin_amdgcn_sched_barrier(0);             // all of them under way before the first is waited for
    };
    Group f0, f1;
    load(first + wave, f0);

    // Tokens, in pieces of 16 bytes, permuted within a chunk by the row's number (see below); a wavefront has four chunks (eight) of a row at a time.
    {
        const uint32_t x_ld = (uint32_t)(XT == kXBf16 ? 2 * a.ld_x : a.k), row_bytes = (uint32_t)(XT == kXBf16 ? 2 * a.k : a.k);
        const void* base = XT == kXBf16 ? a.x : a.x_codes;
        const i32x4 words = buffer_words(base, (uint32_t)m_last * x_ld + row_bytes);
        const int lds_row = a.chunks_each * kRow, turns = (lds_row + 1023) / 1024;      // of 64 pieces
        for (int q = wave; q < (m_last + 1) * turns; q += kWaves) {
            const int row = q / turns, at = (q - row * turns) * 1024 + lane * 16;
            const uint32_t from = (uint32_t)first * kRow + (uint32_t)(at / kRow) * kRow + piece_of<XT == kXBf16 ? (int)kXBf16 : (int)kXMx>(row, at % kRow / 16) * 16u;
            const bool in = at < lds_row && from < row_bytes;
            // lanes behind the end of the row's part stay out
            if (at < lds_row) load_to_lds(words, in ? from + (uint32_t)row * x_ld : kNowhere, 0, lds_of(&xs[row * lds_row + (q - row * turns) * 1024]));
        }
        if constexpr (XT != kXBf16) {
            const __amdgpu_buffer_rsrc_t b = buffer_of(a.x_scales, (uint32_t)(m_last + 1) * (uint32_t)(a.k / 32));
            for (int q = threadIdx.x; q < (m_last + 1) * a.chunks_each; q += 64 * kWaves) {
                const int row = q / a.chunks_each, chunk = first + q - row * a.chunks_each;
                uint32_t v = 0;
                if (chunk * 128 + 128 <= a.k) {
                    v = buffer_load_scales<8>(b, (uint32_t)(row * (a.k / 32) + chunk * 4), 0);
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        v |= buffer_load_scales<32>(b, chunk * 128 + 32 * i < a.k ? (uint32_t)(row * (a.k / 32) + chunk * 4 + i) : kNowhere, 0) << (8 * i);
                }
                x_scales[q] = v;
            }
        }
    }
    // Scales of W: rows of words, an odd number of them so that 16 rows lie in 16 banks.
    const int s_bytes = (a.chunks_each * 128) >> shift, s_words = (s_bytes + 3) / 4, s_row = s_words | 1;
    {
        const int s_first = (first * 128) >> shift;
        const __amdgpu_buffer_rsrc_t b = buffer_of(a.w_scales + (int64_t)n0 * per_row, (uint32_t)(n_last + 1) * (uint32_t)per_row);
        const bool words_whole = (per_row & 3) == 0;   // the parts begin at multiples of four bytes
        for (int q = threadIdx.x; q < (n_last + 1) * s_words; q += 64 * kWaves) {
            const int row = q / s_words, at = s_first + 4 * (q - row * s_words);
            uint32_t v = 0;
            if (words_whole) {
                v = buffer_load_scales<8>(b, at < per_row ? (uint32_t)(row * per_row + at) : kNowhere, 0);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v |= buffer_load_scales<32>(b, at + i < per_row ? (uint32_t)(row * per_row + at + i) : kNowhere, 0) << (8 * i);
            }
            w_scales[row * s_row + (at - s_first) / 4] = v;
        }
    }
    all_loads_done();
    __syncthreads();

    const ScaleReader scale_of(a.scale_fmt);
    f32x4 acc[MT][NT] = {};
    auto multiply = [&](int c0, const Group& f) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int chunk = c0 + u * kWaves;
            if (chunk >= end) break;                   // the same for all lanes
            const int c = chunk - first;
            uint32_t s[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const uint8_t* p = reinterpret_cast<const uint8_t*>(&w_scales[min(16 * i + r16, n_last) * s_row]) + (((c * 128) + 32 * g) >> shift);
                if constexpr (SB == 8) s[i] = *reinterpret_cast<const uint32_t*>(p);
                else if constexpr (SB == 16) s[i] = *reinterpret_cast<const uint16_t*>(p);
                else s[i] = *p;
            }
            const uint8_t* xrow[MT];
            uint32_t xscale[MT], row[MT];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                row[t] = (uint32_t)min(16 * t + r16, m_last);
                xrow[t] = &xs[(row[t] * a.chunks_each + c) * kRow];
                if constexpr (XT != kXBf16) xscale[t] = x_scales[row[t] * a.chunks_each + c] >> (8 * g);
            }
            if constexpr (XT == kXMx) {
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    // v_mfma_scale_f32_16x16x128_f8f6f4: FP4 has 32 consecutive k a group, E4M3 16 at 16 g and 16 at 64 + 16 g; the
                    // scale of a group's 32 k comes from that group's lanes for both.
                    const uint4 lo = *reinterpret_cast<const uint4*>(xrow[t] + piece_of<kXMx>(row[t], g) * 16);
                    const uint4 hi = *reinterpret_cast<const uint4*>(xrow[t] + piece_of<kXMx>(row[t], 4 + g) * 16);
                    const i32x8 x = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const i32x8 w = {(int)f.c[u][i].x, (int)f.c[u][i].y, (int)f.c[u][i].z, (int)f.c[u][i].w, 0, 0, 0, 0};
                        acc[t][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc[t][i], 4, 0, 0, (int)s[i], 0, (int)xscale[t]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint4 x[MT];
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        if constexpr (XT == kXBf16) {
                            x[t] = *reinterpret_cast<const uint4*>(xrow[t] + piece_of<kXBf16>(row[t], 4 * g + j) * 16);
                        } else {
                            const uint2 v8 = *reinterpret_cast<const uint2*>(xrow[t] + piece_of<kXMx>(row[t], 2 * g + j / 2) * 16 + 8 * (j & 1));
                            float v[8];
                            q8_widen(v8, q8_scale(xscale[t] & 255u), v);
                            x[t] = bf16_of8(v);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const uint32_t cc = j == 0 ? f.c[u][i].x : j == 1 ? f.c[u][i].y : j == 2 ? f.c[u][i].z : f.c[u][i].w;
                        const uint32_t byte = (SB == 8) ? (s[i] >> (8 * j)) & 255u : (SB == 16) ? (s[i] >> (8 * (j / 2))) & 255u : s[i];
                        const uint4 w = widen_codes(cc, scale_of(byte));
#pragma unroll
                        for (int t = 0; t < MT; ++t) acc[t][i] = mfma_bf16(w, x[t], acc[t][i]);
                    }
                }
            }
        }
    };
    // The next group is on its way while one is multiplied; its loads are not conditional (beyond the end they give zeros), or the
    // compiler would wait for all of them.  Where the wavefronts have one group each, there is no next one.
    constexpr int kStep = kWaves * AHEAD;
    if (end - first <= kStep) {
        multiply(first + wave, f0);
    } else {
        for (int c0 = first + wave; c0 < end; c0 += 2 * kStep) {
            load(c0 + kStep, f1);
            multiply(c0, f0);
            load(c0 + 2 * kStep, f0);
            multiply(c0 + kStep, f1);
        }
    }
    __syncthreads();                                   // nobody reads tokens any more
    f32x4* sums = reinterpret_cast<f32x4*>(xs);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < NT; ++i) sums[(wave * (NT * MT) + t * NT + i) * 64 + lane] = acc[t][i];
    __syncthreads();
    for (int q = wave; q < NT * MT; q += kWaves) {
        f32x4 v = sums[q * 64 + lane];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += sums[(w * (NT * MT) + q) * 64 + lane];
        const int n = n0 + 16 * (q % NT), m = 16 * (q / NT);
        if (a.parts) {
            if (m < a.m && n < a.n) part_tile(a, blockIdx.z, m, n)[lane] = v;
        } else {
            store_y(a, m + r16, n + 4 * g, v * (a.t_dev ? *a.t_dev : a.T));
        }
    }
}

// Adds up the parts of k of a few tokens, and their adapters, each lane for its token, however many different adapters the tokens have (24
// tokens with 12 adapters, 7 parts: one adapter after the other 12.7 us, so 6.0; 3.9 without).  A wavefront has one tile.  Bound by its
// trips to memory, one behind the other: a part of k, then the next, then the parts of the inner product.
__global__ void __launch_bounds__(256) linear_join_few_kernel(LinearArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = (blockIdx.x * 4 + wave) * 16, m0 = blockIdx.y * 16;
    if (n0 >= a.n) return;
    const int m = m0 + (lane & 15), n = n0 + 4 * (lane >> 4);
    f32x4 acc = {};
    for (int s = 0; s < a.splits; ++s) acc += part_tile(a, s, m0, n0)[lane];
    acc *= a.t_dev ? *a.t_dev : a.T;
    const int id = a.rank > 0 ? adapter_of(a, m) : -1;
    if (id >= 0) {
        for (int r = 0; r < a.rank; r += 8) {
            float u[8];
            load8<kF32>(a.low, (int64_t)m * a.rank + r, u);
            for (int p = 1; p < a.low_parts; ++p) {
                float more[8];
                load8<kF32>(a.low, ((int64_t)p * a.m + m) * a.rank + r, more);
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] += more[i];
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float b[8];
                load8<kBF16>(a.b, ((int64_t)id * a.n + min(n + q, a.n - 1)) * a.rank + r, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[q] = __builtin_fmaf(u[i], b[i], acc[q]);
            }
        }
    }
    store_y(a, m, n, acc);
}

// Adds up the parts of k, and the adapters.  A wavefront has 16 tokens and NT tiles of 16 columns.  Bound by memory: two parts of 2048 x
// 4096 (67 MB in, 17 out) 15.8 us, with 8 adapters in order 23.4, mixed (6.5 to a tile) 49.5.
template <int NT>
__global__ void __launch_bounds__(256) linear_join_kernel(LinearArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = (blockIdx.x * 4 + wave) * (16 * NT), m0 = blockIdx.y * 16;
    if (n0 >= a.n) return;
    f32x4 acc[NT] = {};
    for (int s = 0; s < a.splits; ++s)
#pragma unroll
        for (int i = 0; i < NT; ++i)
            if (n0 + 16 * i < a.n) acc[i] += part_tile(a, s, m0, n0 + 16 * i)[lane];
    const float T = a.t_dev ? *a.t_dev : a.T;
#pragma unroll
    for (int i = 0; i < NT; ++i) acc[i] *= T;
    const int m = m0 + (lane & 15);
    if (a.rank > 0) add_adapters<NT>(a, m, n0, acc);
#pragma unroll
    for (int i = 0; i < NT; ++i) store_y(a, m, n0 + 16 * i + 4 * (lane >> 4), acc[i]);
}

// ---------------------------------------------------------------------------------------
// Many tokens: tiles of BN rows of W times BM tokens, eight wavefronts, k in chunks of 128.  Tokens, codes and scales all go through LDS,
// straight from memory but for Q8 that is widened (its tokens pass through registers, where they become bf16).  LDS has STAGES chunks in
// turn; the codes have one buffer where it has no room for more.  Codes are widened behind LDS, by the wavefronts that multiply them.
// LDS rows of tokens are 256 bytes (bf16) or 128 (Q8 as it is) without padding; 16-byte pieces of a row are permuted by the row number, so
// that the 16 rows of a fragment read 16 (8) different groups of banks.
// What bounds it: the matrix instructions, with the loads and the widening not quite behind them.  4096 x 28672 x 4096, the kernel alone:
// Q8 against E8M0 by the scaled instruction 409 us (2.35 PFLOP/s), widened 960 (1.0); bf16 against E4M3 776 (1.24).
// ---------------------------------------------------------------------------------------
constexpr int kTiledThreads = 512;

// The same for rows of 64 bytes of codes.
__device__ __forceinline__ uint32_t code_piece(uint32_t row, uint32_t piece) { return piece ^ ((row >> 1) & 3u); }

// STAGES - 1 chunks are on their way while one is multiplied.  Where LDS has no room for two chunks of codes beside the tokens
// (tiles of 256 x 256 in bf16), the wavefronts take the chunk's codes into registers first, and the next ones replace them.
template <int XT, int SB, int WN, int WM, int NT, int MT, int STAGES>
__global__ void __launch_bounds__(kTiledThreads, 2) linear_tiled_kernel(LinearArgs a)
{
    constexpr int BN = WN * NT * 16, BM = WM * MT * 16;
    constexpr int kRow = XT == kXMx ? 128 : 256;                        // bytes of a row of the chunk
    constexpr int kPieces = kRow / 16;
    constexpr int kGroup = SB == 8 ? 1 : SB == 16 ? 2 : 4;              // chunks of a group of scales
    constexpr int kGroups = (STAGES - 2) / kGroup + 2;                  // groups in LDS: that of the chunk at hand to that of the furthest ahead
    constexpr int kRoom = 160 * 1024 - STAGES * BM * kRow - kGroups * (BN + (XT == kXMx ? BM : 0)) * 16;
    constexpr int kCodeBuffers = kRoom >= STAGES * BN * 64 ? STAGES : 1;
    static_assert(WN * WM * 64 == kTiledThreads, "eight wavefronts");
    static_assert(STAGES == 2 || (kCodeBuffers == STAGES && XT != kXQ8), "what is not in LDS is one chunk ahead");
    __shared__ __align__(16) uint8_t xs[STAGES][BM * kRow];
    __shared__ __align__(16) uint8_t wcodes[kCodeBuffers][BN * 64];
    __shared__ uint4 wscale[kGroups][BN], xscale[XT == kXMx ? kGroups : 1][XT == kXMx ? BM : 1];     // 16 bytes a row
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r16 = lane & 15;
    const int wn = wave % WN, wm = wave / WN;
    int bx = blockIdx.x, by = blockIdx.y;
    if (gridDim.y >= 8u) {
        // Workgroups go to the eight dies in turn, each with an L2 of its own: a die gets a run of tiles, in strips of four tiles of tokens, so
        // that the 32 it has at a time share 4 tiles of tokens and 8 of W.  2048 x 4096 x 14336 231 -> 223 us, 4096 x 28672 x 4096 in 8 bits
        // 432.5 -> 426.5; with fewer tiles of tokens the order of the grid is as good or better (256 x 4096 x 4096: 25.0 us, 26.2).
        const unsigned total = gridDim.x * gridDim.y, id = blockIdx.x + gridDim.x * blockIdx.y, die = id % 8u;
        const unsigned tile = die * (total / 8u) + min(die, total % 8u) + id / 8u, strip = tile / (4u * gridDim.x);
        const unsigned in_strip = tile - strip * (4u * gridDim.x), high = min(4u, gridDim.y - 4u * strip);
        bx = (int)(in_strip / high);
        by = (int)(4u * strip + in_strip % high);
    }
    const int nb = bx * BN, nw = nb + wn * (NT * 16), m0 = by * BM;
    const int shift = __builtin_ctz(a.block), per_row = a.k >> shift;
    const int first = blockIdx.z * a.chunks_each, chunks = min((a.k + 127) / 128, first + a.chunks_each);

    // scalar bases, 32-bit offsets: the launch sees to it that a tile's rows span less than 4 GiB
    const int n_last = min(a.n - 1 - nb, BN - 1);
    const uint8_t* code_base = a.w_codes + (int64_t)nb * (a.k / 2);
    const uint32_t code_bytes = (uint32_t)(n_last + 1) * (uint32_t)(a.k / 2);
    const i32x4 code_words = buffer_words(code_base, code_bytes);
    const uint8_t* scale_base = a.w_scales + (int64_t)nb * per_row;
    const uint32_t scale_bytes = (uint32_t)(n_last + 1) * (uint32_t)per_row;
    constexpr int kCodeLoads = BN * 64 / (kTiledThreads * 16);
    uint32_t code_at[kCodeLoads];
#pragma unroll
    for (int i = 0; i < kCodeLoads; ++i) {
        const uint32_t place = (uint32_t)(wave * kCodeLoads + i) * 64u + (uint32_t)lane, row = place / 4u;
        code_at[i] = (uint32_t)min((int)row, n_last) * (uint32_t)(a.k / 2) + code_piece(row, place % 4u) * 16u;
    }
    const ScaleReader scale_of(a.scale_fmt);
    f32x4 acc[MT][NT] = {};
    auto start_w = [&](int chunk, int buf) {
        const bool whole = chunk * 128 + 128 <= a.k;
#pragma unroll
        for (int i = 0; i < kCodeLoads; ++i) {
            uint32_t at = code_at[i];
            if (!whole) {
                const uint32_t place = (uint32_t)(wave * kCodeLoads + i) * 64u + (uint32_t)lane;
                at = chunk * 128 + 32 * (int)code_piece(place / 4u, place % 4u) < a.k ? at : kNowhere;
            }
            load_to_lds(code_words, at, chunk * 64, lds_of(&wcodes[buf % kCodeBuffers][(wave * kCodeLoads + i) * 1024]));
        }
    };

    // The activations' chunk: what goes straight to LDS, and what goes through registers (Q8 to be widened, scales, and a last
    // chunk that is not whole, whose missing part is zeros).
    constexpr int kDirect = BM * kRow / (kTiledThreads * 16);           // pieces of 16 bytes a thread
    constexpr int kThreadsARow = kTiledThreads / BM > 0 ? kTiledThreads / BM : 1, kCodes = 128 / kThreadsARow;
    const int m_last = min(a.m - 1 - m0, BM - 1);
    const char* x_base = XT == kXBf16 ? static_cast<const char*>(a.x) + (int64_t)m0 * a.ld_x * 2 : reinterpret_cast<const char*>(a.x_codes) + (int64_t)m0 * a.k;
    const uint32_t x_ld = (uint32_t)(XT == kXBf16 ? 2 * a.ld_x : a.k);
    const uint32_t x_bytes = (uint32_t)m_last * x_ld + (uint32_t)(XT == kXBf16 ? 2 * a.k : a.k);
    const __amdgpu_buffer_rsrc_t x_codes = buffer_of(x_base, x_bytes);
    const i32x4 x_words = buffer_words(x_base, x_bytes);
    const __amdgpu_buffer_rsrc_t x_scales = buffer_of(XT == kXBf16 ? nullptr : a.x_scales + (int64_t)m0 * (a.k / 32), (uint32_t)(m_last + 1) * (uint32_t)(a.k / 32));
    uint32_t x_at[XT == kXQ8 ? 1 : kDirect], scales_at = 0;
    if constexpr (XT == kXQ8) {
        const uint32_t row = (uint32_t)min((int)threadIdx.x / kThreadsARow, m_last), first = (threadIdx.x % kThreadsARow) * kCodes;
        x_at[0] = row * x_ld + first;
        scales_at = row * (uint32_t)(a.k / 32) + first / 32u;
    } else {
#pragma unroll
        for (int i = 0; i < kDirect; ++i) {
            const uint32_t place = (uint32_t)(wave * kDirect + i) * 64u + (uint32_t)lane, row = place / kPieces;
            x_at[i] = (uint32_t)min((int)row, m_last) * x_ld + piece_of<XT>(row, place % kPieces) * 16u;
        }
    }
    uint4 held[XT == kXQ8 ? kCodes / 16 : 1];
    uint32_t held_scales[(kCodes + 31) / 32] = {};
    auto start_x = [&](int chunk, int buf) {
        const int k0 = chunk * 128;
        if constexpr (XT == kXQ8) {
            const int first = k0 + (int)(threadIdx.x % kThreadsARow) * kCodes;
#pragma unroll
            for (int i = 0; i < kCodes / 16; ++i)
                held[i] = buffer_load16(x_codes, first + 16 * i < a.k ? x_at[0] + 16u * i : kNowhere, k0);
#pragma unroll
            for (int i = 0; i < (kCodes + 31) / 32; ++i)
                held_scales[i] = buffer_load_scales<32>(x_scales, first + 32 * i < a.k ? scales_at + (uint32_t)i : kNowhere, k0 / 32);
        } else {
            const bool whole = k0 + 128 <= a.k;
#pragma unroll
            for (int i = 0; i < kDirect; ++i) {
                uint32_t at = x_at[i];
                if (!whole) {
                    const uint32_t place = (uint32_t)(wave * kDirect + i) * 64u + (uint32_t)lane;
                    const int in_row = chunk * kRow + (int)piece_of<XT>(place / kPieces, place % kPieces) * 16;
                    at = in_row < (XT == kXMx ? a.k : 2 * a.k) ? at : kNowhere;
                }
                load_to_lds(x_words, at, chunk * kRow, lds_of(&xs[buf][(wave * kDirect + i) * 1024]));
            }
        }
    };
    // Scales come 16 bytes of a row at a time, enough for kGroup chunks: a lane that loads the few bytes of its chunk touches as many
    // lines for them.  The first wavefronts load those of W, the last ones those of the tokens; straight to LDS where they lie on 16 bytes, else
    // through registers, byte by byte where rows begin anywhere.
    constexpr int kXThreads = kTiledThreads - BM;
    const bool w_thread = wave < BN / 64, x_thread = XT == kXMx && wave >= kXThreads / 64;
    static_assert(BN + (XT == kXMx ? BM : 0) <= kTiledThreads, "one row a thread");
    const int scale_row = w_thread ? min((int)threadIdx.x, n_last) : min((int)threadIdx.x - kXThreads, m_last);
    const int scale_row_bytes = w_thread ? per_row : a.k / 32;
    const bool straight = shift <= 5 && (per_row & 15) == 0 && (reinterpret_cast<uintptr_t>(a.w_scales) & 15u) == 0 &&
                          (XT != kXMx || (reinterpret_cast<uintptr_t>(a.x_scales) & 15u) == 0);       // block 32 where XT is kXMx, or not straight
    const i32x4 scale_words = w_thread ? buffer_words(scale_base, scale_bytes) : buffer_words(XT == kXMx ? a.x_scales + (int64_t)m0 * (a.k / 32) : nullptr, (uint32_t)(m_last + 1) * (uint32_t)(a.k / 32));
    const __amdgpu_buffer_rsrc_t scales = buffer_of(w_thread ? scale_base : XT == kXMx ? a.x_scales + (int64_t)m0 * (a.k / 32) : nullptr,
                                                    w_thread ? scale_bytes : (uint32_t)(m_last + 1) * (uint32_t)(a.k / 32));
    uint4 group = make_uint4(0u, 0u, 0u, 0u);
    auto group_of = [&](int chunk) { return (chunk - first) / kGroup % kGroups; };
    auto start_scales = [&](int chunk) {
        if (!w_thread && !x_thread) return;
        const int at = w_thread ? (chunk * 128) >> shift : chunk * 4;
        if (straight) {
            const uint4* to = w_thread ? &wscale[group_of(chunk)][wave * 64] : &xscale[XT == kXMx ? group_of(chunk) : 0][wave * 64 - kXThreads];
            load_to_lds(scale_words, (uint32_t)(scale_row * scale_row_bytes), at, lds_of(to));
        } else if ((scale_row_bytes & 3) == 0) {
            group = buffer_load16(scales, (uint32_t)(scale_row * scale_row_bytes + at), 0);
        } else {
            uint32_t v[4] = {};
#pragma unroll
            for (int i = 0; i < 16; ++i)
                v[i / 4] |= buffer_load_scales<32>(scales, at + i < scale_row_bytes ? (uint32_t)(scale_row * scale_row_bytes + at + i) : kNowhere, 0) << (8 * (i % 4));
            group = make_uint4(v[0], v[1], v[2], v[3]);
        }
    };
    auto finish_scales = [&](int chunk) {
        if (straight) return;
        if (w_thread) wscale[group_of(chunk)][threadIdx.x] = group;
        else if (x_thread) xscale[XT == kXMx ? group_of(chunk) : 0][threadIdx.x - kXThreads] = group;
    };
    auto finish_x = [&](int buf) {
        if constexpr (XT == kXQ8) {
            const uint32_t row = threadIdx.x / kThreadsARow, first = (threadIdx.x % kThreadsARow) * kCodes;
#pragma unroll
            for (int i = 0; i < kCodes / 16; ++i) {
                const float S = q8_scale(held_scales[i / 2]);
                float v[8];
                q8_widen(make_uint2(held[i].x, held[i].y), S, v);
                *reinterpret_cast<uint4*>(&xs[buf][row * kRow + piece_of<XT>(row, first / 8 + 2 * i) * 16]) = bf16_of8(v);
                q8_widen(make_uint2(held[i].z, held[i].w), S, v);
                *reinterpret_cast<uint4*>(&xs[buf][row * kRow + piece_of<XT>(row, first / 8 + 2 * i + 1) * 16]) = bf16_of8(v);
            }
        }
    };
    auto x_piece = [&](int buf, int t, int piece) {
        const uint32_t row = wm * (MT * 16) + t * 16 + r16;
        return *reinterpret_cast<const uint4*>(&xs[buf][row * kRow + piece_of<XT>(row, piece) * 16]);
    };

    auto start = [&](int chunk, int buf) {
        if ((chunk - first) % kGroup == 0) start_scales(chunk);
        start_x(chunk, buf);
        start_w(chunk, buf);
    };
    auto finish = [&](int chunk, int buf) {
        if ((chunk - first) % kGroup == 0) finish_scales(chunk);
        finish_x(buf);
    };
    auto step = [&](int chunk, auto buf_constant) {
        constexpr int buf = decltype(buf_constant)::value, ahead = (buf + STAGES - 1) % STAGES;
        // The loads of the chunks after this one may be under way still (those of scales count too: then this waits for more than it needs).
        if (STAGES > 2 && chunk + STAGES - 2 < chunks) loads_done_but<(STAGES - 2) * (kDirect + kCodeLoads)>();
        else all_loads_done();
        __syncthreads();                      // this chunk is in LDS, and nobody reads the one before any more
        const int next = chunk + STAGES - 1;
        if (kCodeBuffers == STAGES && next < chunks) start(next, ahead);
        struct { uint4 c[NT]; } w;
        uint32_t s[NT];
        const int sbuf = group_of(chunk), group_first = chunk - (chunk - first) % kGroup;
        const int s_at = ((chunk * 128 + 32 * g) >> shift) - ((group_first * 128) >> shift);
        const bool in = chunk * 128 + 32 * g < a.k;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const uint32_t row = wn * (NT * 16) + 16 * i + r16;
            w.c[i] = *reinterpret_cast<const uint4*>(&wcodes[buf % kCodeBuffers][row * 64u + code_piece(row, g) * 16u]);
            const uint8_t* p = reinterpret_cast<const uint8_t*>(&wscale[sbuf][row]) + s_at;
            if constexpr (SB == 8) s[i] = *reinterpret_cast<const uint32_t*>(p);
            else if constexpr (SB == 16) s[i] = *reinterpret_cast<const uint16_t*>(p);
            else s[i] = *p;
            s[i] = in ? s[i] : 0u;            // behind the end of a row: what follows it
        }
        if constexpr (kCodeBuffers == 1) {
            __syncthreads();                  // everybody has its codes: the next ones may come
            if (next < chunks) start(next, ahead);
        }
        const uint8_t* xscale_bytes = reinterpret_cast<const uint8_t*>(&xscale[XT == kXMx ? sbuf : 0][0]) + (XT == kXMx ? (wm * (MT * 16) + r16) * 16 + 4 * (chunk - group_first) + g : 0);
        auto x_scale = [&](int t) { return in ? (uint32_t)xscale_bytes[t * 256] : 0u; };
        // One fragment of activations ahead of the products, and not more: the compiler would load them all first.
        if constexpr (XT == kXMx) {
            uint4 lo = x_piece(buf, 0, g), hi = x_piece(buf, 0, 4 + g);
            uint32_t xscales = x_scale(0);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const i32x8 x = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
                const uint32_t xs_now = xscales;
                if (t + 1 < MT) {
                    lo = x_piece(buf, t + 1, g);
                    hi = x_piece(buf, t + 1, 4 + g);
                    xscales = x_scale(t + 1);
                }
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const i32x8 v = {(int)w.c[i].x, (int)w.c[i].y, (int)w.c[i].z, (int)w.c[i].w, 0, 0, 0, 0};
                    acc[t][i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v, x, acc[t][i], 4, 0, 0, (int)s[i], 0, (int)xs_now);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            uint4 x = x_piece(buf, 0, 4 * g);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint4 v[NT];
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const uint32_t cc = j == 0 ? w.c[i].x : j == 1 ? w.c[i].y : j == 2 ? w.c[i].z : w.c[i].w;
                    const uint32_t byte = (SB == 8) ? (s[i] >> (8 * j)) & 255u : (SB == 16) ? (s[i] >> (8 * (j / 2))) & 255u : s[i];
                    v[i] = widen_codes(cc, scale_of(byte));
                }
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const uint4 now = x;
                    if (t + 1 < MT) x = x_piece(buf, t + 1, 4 * g + j);
                    else if (j + 1 < 4) x = x_piece(buf, 0, 4 * g + j + 1);
#pragma unroll
                    for (int i = 0; i < NT; ++i) acc[t][i] = mfma_bf16(v[i], now, acc[t][i]);
                    __builtin_amdgcn_sched_barrier(6);         // but for vector and scalar arithmetic: codes are widened between the products
                }
            }
        }
        finish(next, ahead);                  // behind the last chunk: of nothing, to places that nobody reads
    };

#pragma unroll
    for (int c = 0; c < STAGES - 1; ++c)
        if (first + c < chunks) {
            start(first + c, c);
            finish(first + c, c);
        }
    for (int chunk = first; chunk < chunks; chunk += STAGES) {
        step(chunk, std::integral_constant<int, 0>());
        if (chunk + 1 < chunks) step(chunk + 1, std::integral_constant<int, 1>());
        if constexpr (STAGES > 2)
            if (chunk + 2 < chunks) step(chunk + 2, std::integral_constant<int, 2>());
        if constexpr (STAGES > 3)
            if (chunk + 3 < chunks) step(chunk + 3, std::integral_constant<int, 3>());
    }
    if (a.parts) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int m = m0 + wm * (MT * 16) + t * 16, n = nw + 16 * i;
                if (m < a.m && n < a.n) part_tile(a, blockIdx.z, m, n)[lane] = acc[t][i];
            }
        return;
    }
    const float T = a.t_dev ? *a.t_dev : a.T;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = m0 + wm * (MT * 16) + t * 16 + r16;
#pragma unroll
        for (int i = 0; i < NT; ++i) acc[t][i] *= T;
        if (a.rank > 0) add_adapters<NT>(a, m, nw, acc[t]);
#pragma unroll
        for (int i = 0; i < NT; ++i) store_y(a, m, nw + 16 * i + 4 * g, acc[t][i]);
    }
}

// y = 0, for contractions of no length.
__global__ void __launch_bounds__(256) zero_rows_kernel(LinearArgs a)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n >= a.n) return;
    for (int64_t m = blockIdx.y; m < a.m; m += gridDim.y) {
        if (a.y_dtype == kBF16) static_cast<uint16_t*>(a.y)[m * a.ld_y + n] = 0;
        else static_cast<float*>(a.y)[m * a.ld_y + n] = 0.0f;
    }
}

// Whether Q8 and the weights multiply as they are.  The scaled matrix instruction sums its 128 products with about 21 bits of the
// largest (error against 64 bits, 2-norm: 4.2e-6, fp32 sums of widened elements 3e-7): a bf16 output (1.7e-3) shows that where its terms
// cancel, so it is the caller's choice; an fp32 output would show it everywhere and is widened.
bool scaled_products(const LinearArgs& a)
{
    return a.mx_sums && a.x_codes && a.scale_fmt == kE8M0 && a.block >= 32 && a.y_dtype == kBF16;
}

LinearPlan plan_of(const LinearArgs& a) { return plan_linear({a.m, a.n, a.k, a.block, a.x != nullptr, scaled_products(a), a.rank}); }

template <int XT, int SB, int WN, int WM, int NT, int MT, int STAGES>
void launch_tiled(const LinearArgs& a, const LinearPlan& p, hipStream_t stream)
{
    constexpr int BN = WN * NT * 16, BM = WM * MT * 16;
    hipLaunchKernelGGL((linear_tiled_kernel<XT, SB, WN, WM, NT, MT, STAGES>),
                       dim3((unsigned)((a.n + BN - 1) / BN), (unsigned)((a.m + BM - 1) / BM), (unsigned)p.splits), dim3(kTiledThreads), 0, stream, a);
}

template <int XT, int SB, int NT, int MT, int AHEAD>
void launch_direct(const LinearArgs& a, const LinearPlan& p, hipStream_t stream)
{
    const int main = (a.n + 16 * NT - 1) / (16 * NT);
    const DirectLds lds = direct_lds({a.m, a.n, a.k, a.block, XT == kXBf16, XT == kXMx, a.rank}, NT, MT, p.chunks_each);
    hipLaunchKernelGGL((linear_direct_kernel<XT, SB, NT, MT, AHEAD>), dim3((unsigned)(a.low_blocks + main), 1, (unsigned)p.splits),
                       dim3(64 * kWaves), lds.bytes, stream, a, main, lds);
}

template <int XT, int SB>
hipError_t launch_products(const LinearArgs& a, const LinearPlan& p, hipStream_t stream)
{
    if (p.tiled) {
        // Wavefronts beside each other in n where elements are widened, so that no code is widened twice (256 x 256: 831 -> 796 us at 4096 x
        // 28672 x 4096); in two rows where they multiply as they are, which reads less of LDS.
        constexpr bool kWide = XT != kXMx;
        if constexpr (!kWide)
            if (p.mt == 8) {
                launch_tiled<XT, SB, 4, 2, 4, 4, 3>(a, p, stream);
                return hipGetLastError();
            }
        if (p.mt == 16) launch_tiled<XT, SB, kWide ? 8 : 4, kWide ? 1 : 2, kWide ? 2 : 4, kWide ? 16 : 8, 2>(a, p, stream);
        else if (p.nt == 16) launch_tiled<XT, SB, kWide ? 8 : 4, kWide ? 1 : 2, kWide ? 2 : 4, kWide ? 4 : 2, kWide ? 2 : 4>(a, p, stream);
        else launch_tiled<XT, SB, kWide ? 8 : 4, kWide ? 1 : 2, kWide ? 1 : 2, kWide ? 4 : 2, kWide ? 2 : 4>(a, p, stream);
    } else {
        // one chunk ahead; two where it is 16 rows (4096 x 14336, one token: 11.6 -> 10.8 us; four 11.6; 64 rows, two 14.1, one 13.9)
        if constexpr (XT != kXBf16)                            // bf16 of more than 16 tokens goes to tiles
            if (p.mt == 2) {
                launch_direct<XT, SB, 4, 2, 1>(a, p, stream);
                return hipGetLastError();
            }
        if (p.nt == 4) launch_direct<XT, SB, 4, 1, 1>(a, p, stream);
        else if (p.nt == 2) launch_direct<XT, SB, 2, 1, 1>(a, p, stream);
        else launch_direct<XT, SB, 1, 1, 2>(a, p, stream);
    }
    return hipGetLastError();
}

template <int XT>
hipError_t launch_by_block(const LinearArgs& a, const LinearPlan& p, hipStream_t stream)
{
    if (a.block == 8) return launch_products<XT, 8>(a, p, stream);
    if (a.block == 16) return launch_products<XT, 16>(a, p, stream);
    return launch_products<XT, 32>(a, p, stream);
}

// Rows [first, first + count) of a call.
LinearArgs rows_of(const LinearArgs& a, int64_t first, int64_t count)
{
    LinearArgs p = a;
    p.m = (int)count;
    if (a.x) p.x = static_cast<const uint16_t*>(a.x) + first * a.ld_x;
    if (a.x_codes) { p.x_codes += first * a.k; p.x_scales += first * (a.k / 32); }
    if (a.ids) p.ids += first;
    p.y = static_cast<char*>(a.y) + first * a.ld_y * (a.y_dtype == kBF16 ? 2 : 4);
    return p;
}

hipError_t launch_rows(LinearArgs a, void* workspace, hipStream_t stream)
{
    const LinearPlan p = plan_of(a);
    a.splits = p.splits;
    a.chunks_each = p.chunks_each;
    a.low = static_cast<float*>(workspace);
    a.parts = p.join ? reinterpret_cast<float*>(static_cast<char*>(workspace) + p.low_bytes) : nullptr;
    a.low_parts = p.low_parts;
    a.low_slots = a.ids ? (a.count < 16 ? a.count : 16) : 1;
    a.low_blocks = 0;
    if (a.rank > 0) {
        const unsigned blocks = (unsigned)((a.m + 15) / 16 * ((a.rank + 15) / 16) * a.low_parts * a.low_slots);
        if (p.tiled) {
            if (a.x) hipLaunchKernelGGL(lowrank_kernel<kXBf16>, dim3(blocks), dim3(64 * kWaves), 0, stream, a);
            else hipLaunchKernelGGL(lowrank_kernel<kXQ8>, dim3(blocks), dim3(64 * kWaves), 0, stream, a);
        } else {
            a.low_blocks = (int)blocks;
        }
    }
    hipError_t e;
    if (a.x) e = launch_by_block<kXBf16>(a, p, stream);
    else if (scaled_products(a)) e = launch_products<kXMx, 32>(a, p, stream);
    else e = launch_by_block<kXQ8>(a, p, stream);
    if (e == hipSuccess && p.join) {
        const unsigned rows = (unsigned)((a.m + 15) / 16);
        if (a.m > 64) hipLaunchKernelGGL(linear_join_kernel<4>, dim3((unsigned)((a.n + 255) / 256), rows), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL(linear_join_few_kernel, dim3((unsigned)((a.n + 63) / 64), rows), dim3(256), 0, stream, a);
        e = hipGetLastError();
    }
    return e;
}

int64_t rows_a_launch(const LinearArgs& a) { return a.x ? linear_rows_a_launch(a.m, a.ld_x) : kMostRows; }

}  // namespace

size_t linear_workspace(const LinearArgs& a)
{
    const int64_t most = rows_a_launch(a);
    LinearArgs piece = a;
    piece.m = (int)(a.m < most ? a.m : most);
    const LinearPlan p = plan_of(piece);
    size_t bytes = p.low_bytes + p.part_bytes;
    if (a.m > most && a.m % most != 0) {                   // the last rows are cut up otherwise
        piece.m = (int)(a.m % most);
        const LinearPlan q = plan_of(piece);
        if (q.low_bytes + q.part_bytes > bytes) bytes = q.low_bytes + q.part_bytes;
    }
    return bytes;
}

hipError_t launch_linear(const LinearArgs& all, void* workspace, hipStream_t stream)
{
    if (all.k == 0) {
        hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)((all.n + 255) / 256), (unsigned)(all.m < 16384 ? all.m : 16384)), dim3(256), 0, stream, all);
        return hipGetLastError();
    }
    const int64_t most = rows_a_launch(all);
    for (int64_t first = 0; first < all.m; first += most) {
        const hipError_t e = launch_rows(rows_of(all, first, all.m - first < most ? all.m - first : most), workspace, stream);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace mxq
