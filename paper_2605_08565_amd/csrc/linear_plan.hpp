// How a call of mxq_linear is cut into workgroups: plain C++, so that it can be checked without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace mxq {

constexpr int kLinearWaves = 8;                            // of the direct kernel's workgroups
constexpr int kScaleBytes = 16 * 1024;                     // LDS of a direct workgroup for scales of W, without the padding of its rows
constexpr int kTokenBytes = 128 * 1024;                    // and for tokens, at most
constexpr int kUnits = 256;                                // compute units

struct LinearShape {
    int m, n, k, block;
    bool bf16;                                             // activations, else Q8
    bool scaled;                                           // Q8 multiplied as it is
    int rank;                                              // 0: no adapters
};

struct LinearPlan {
    bool tiled;                                            // else the direct kernel, all tokens in a workgroup
    int nt, mt;                                            // tiles of 16 rows of W and of 16 tokens a workgroup
    int splits, chunks_each;                               // parts of k, and the chunks of 128 in one
    int low_parts;                                         // parts of k of the adapters' first product
    bool join;                                             // a last launch adds up parts (and the adapters)
    size_t low_bytes, part_bytes;                          // of the workspace
};

// Rows of one launch over bf16 rows ld elements apart: a grid's second side is short, and the rows of a workgroup span at most 2 GiB (32-bit
// offsets).  256 rows of a tile do so below a stride of 2^22, the 16 of the direct kernel below 2^26 (the last tokens of prompts of
// 1024 x 4096 and more; 16 of them by 14336 x 4096 one by one 158 us, together 14.6).  Beyond, rows go one by one.
constexpr int64_t kMostRows = (int64_t)1 << 19;

inline int64_t linear_rows_a_launch(int64_t m, int64_t ld)
{
    if (m <= 1 || ld < (int64_t)1 << 22) return kMostRows;
    return ld < (int64_t)1 << 26 ? 16 : 1;
}

// LDS of a workgroup of the direct kernel: tokens first, which the sums of its wavefronts replace later.
struct DirectLds { int x_scales, w_scales, bytes; };

inline DirectLds direct_lds(const LinearShape& a, int nt, int mt, int chunks_each)
{
    const int x = a.m * chunks_each * (a.bf16 ? 256 : 128), sums = kLinearWaves * nt * mt * 1024;
    const int words = (int)((((int64_t)chunks_each * 128 / a.block + 3) / 4) | 1);            // of a row of scales, an odd number
    DirectLds l;
    l.x_scales = x > sums ? x : sums;
    l.w_scales = l.x_scales + (a.bf16 ? 0 : a.m * chunks_each * 4);
    l.bytes = l.w_scales + 16 * nt * words * 4;
    return l;
}

// Tiles of the tiled kernel, and what a chunk of 128 of one takes on a unit, in us: alone there, and beside others (for bf16; widened Q8
// takes a quarter more in each and goes by the same table).  Measured at
// 4096 x 28672 x 4096, 512 x 14336 x 4096, 128 x 14336 x 4096 and 64 x 14336 x 4096 (bf16 against E4M3) and 4096 x 28672 x 4096 and 512 x 4096 x 4096
// (scaled).
struct LinearTile {
    int nt, mt;
    float alone, beside;
};
// Widened, 256 x 128 takes 2.3 us, more than two of 256 x 64: there is no such kernel.
constexpr LinearTile kWidened[3] = {{16, 16, 3.6f, 3.6f}, {16, 4, 1.4f, 1.13f}, {8, 4, 0.87f, 0.75f}};
constexpr LinearTile kScaled[4] = {{16, 16, 2.0f, 2.0f}, {16, 8, 1.1f, 1.1f}, {16, 4, 0.8f, 0.7f}, {8, 4, 0.55f, 0.42f}};

inline LinearPlan plan_linear(const LinearShape& a)
{
    LinearPlan p = {};
    const int chunks = (a.k + 127) / 128;
    // 24 tokens, 14336 x 4096 bf16: direct 26 us, tiles 18; 4096 x 14336 scaled: 12.9 and 16.4.  Q8 that is widened, as long as 64 rows of W a
    // workgroup make one round on the units (E8M0 block 32, direct and tiles): 4096 x 14336 17.4 and 26.2, 14336 x 4096 15.8 and 19.9, 1024 x 1024
    // 6.4 and 10.3; beyond, 28672 x 4096: 30.2 and 28.1.
    p.tiled = a.m > (a.scaled || (!a.bf16 && a.n <= 64 * kUnits) ? 32 : 16);
    int64_t groups = 1;
    int most = 1, fit = chunks;                            // parts of k at most, chunks in one at most
    int64_t splits = 1;
    if (p.tiled) {
        // The cut that takes least: rounds of workgroups on the units, and for more than one part of k the sums that are written and read.
        float least = 0.0f;
        const LinearTile* const tile = a.scaled ? kScaled : kWidened;
        for (int i = 0; i < (a.scaled ? 4 : 3); ++i) {
            const LinearTile& t = tile[i];
            const int64_t tiles = (int64_t)((a.n + 16 * t.nt - 1) / (16 * t.nt)) * ((a.m + 16 * t.mt - 1) / (16 * t.mt));
            for (int s = 1; s <= 8 && (s == 1 || 4 * s <= chunks); ++s) {
                const int64_t rounds = (tiles * s + kUnits - 1) / kUnits;
                const float each = (float)((chunks + s - 1) / s);
                const float us = each * (rounds == 1 ? t.alone : (float)rounds * t.beside) + (s > 1 ? 4.0f + (float)s * (float)a.m * (float)a.n * 1e-6f : 0.0f);
                if (p.mt == 0 || us < least) {
                    least = us;
                    p.nt = t.nt;
                    p.mt = t.mt;
                    splits = s;
                }
            }
        }
    } else {
        // All tokens of a part of k fit into LDS, and its scales of W do.  Rows of W a workgroup: with few tokens many small workgroups
        // keep loads under way while others multiply; with more, the tokens are loaded into LDS too often.  16 / 32 / 64 rows, 14336 x
        // 4096 E4M3: one token 10.3 / 10.2 / 12.0 us, 8 tokens 14.0 / 11.4 / 13.3, 16 tokens 21 / 17.3 / 14.7.
        const int row = a.bf16 ? 256 : 128;                // bytes of a chunk of a token
        p.mt = a.m > 16 ? 2 : 1;
        p.nt = a.m <= 4 ? 1 : a.m <= 12 ? 2 : 4;
        groups = (a.n + 16 * p.nt - 1) / (16 * p.nt);
        const int scale_chunk = 128 / (a.block > 32 ? 32 : a.block);        // bytes, at most
        const int fit_x = kTokenBytes / (a.m * row), fit_s = kScaleBytes / (16 * p.nt * scale_chunk);
        fit = fit_x < fit_s ? fit_x : fit_s;
        most = chunks / kLinearWaves;
    }
    if (!p.tiled) {
        // one workgroup a unit; with the adapters' workgroups beside them nearly two (24 x 4096 x 14336, 12 adapters, scaled: 4 parts 23.2 us,
        // 7 21.6, 10 22.5; one size, and a kernel of which two lie on a unit: of widened Q8 for more than 16 tokens one does, 30.5 and 32.3).  Adapters behind a product of their own, without the last launch: 16 x 14336 x 4096 18.5 us against 14.2.
        const int64_t want = (a.rank > 0 ? kUnits * 7 / 4 : kUnits) / groups;
        splits = want < most ? want : most;
        if (splits < 1) splits = 1;
    }
    p.chunks_each = (int)((chunks + splits - 1) / splits);
    if (p.chunks_each > fit) p.chunks_each = fit;
    if (p.chunks_each < chunks) {                          // parts begin at whole words of scale bytes
        p.chunks_each &= ~3;
        if (p.chunks_each < 4) p.chunks_each = 4;
    }
    p.splits = (chunks + p.chunks_each - 1) / p.chunks_each;
    p.join = p.splits > 1 || (!p.tiled && a.rank > 0);
    if (a.rank > 0) {
        // about 512 workgroups, with at least 1024 elements of k each; not more than 4 parts where many tokens add them up (one token, k = 14336: 4
        // parts 14.3 us, 8 13.5; 24 tokens 21.6 and 24.0)
        const int64_t tiles = (int64_t)((a.m + 15) / 16) * ((a.rank + 15) / 16), cap = a.m <= 8 ? 8 : 4;
        int64_t parts = 512 / tiles < cap ? 512 / tiles : cap;
        if (parts > a.k / 1024) parts = a.k / 1024;
        p.low_parts = parts < 1 ? 1 : (int)parts;
        p.low_bytes = ((size_t)p.low_parts * a.m * a.rank * sizeof(float) + 255) / 256 * 256;
    }
    if (p.join) p.part_bytes = (size_t)p.splits * ((a.m + 15) / 16) * ((a.n + 15) / 16) * 1024;
    return p;
}

}  // namespace mxq
