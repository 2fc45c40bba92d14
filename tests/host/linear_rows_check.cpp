// Rows of a launch of a projection (csrc/linear_plan.hpp) against the 32-bit offsets of its kernels: the last byte of the rows that one
// workgroup has lies within 2 GiB, far below the offset that stands for nowhere, and as many rows go together as the direct kernel takes.
#include <cmath>
#include <cstdio>
#include <random>

#include "../../paper_2605_08565_amd/csrc/linear_plan.hpp"

using namespace mxq;

int main()
{
    std::mt19937 rng(1);
    const auto upto = [&](double most) { return (int64_t)std::exp(std::uniform_real_distribution<double>(0.0, std::log(most))(rng)); };
    long bad = 0, cases = 0;
    for (int i = 0; i < 1000000; ++i) {
        const int64_t k = 32 * upto((1 << 22) / 32 - 1), m = upto(1 << 20);
        int64_t ld = i % 3 == 0 ? ((int64_t)1 << (20 + i % 9)) + (i % 5 - 2) * 8 : 8 * upto(1 << 26);
        if (ld < k) ld = k;
        const int64_t rows = linear_rows_a_launch(m, ld), together = m < rows ? m : rows;
        bool ok = rows >= 1 && rows <= kMostRows;
        const LinearPlan p = plan_linear({(int)together, 4096, (int)k, 32, true, false, 0});
        const int64_t span = p.tiled ? 16 * p.mt : together;                               // rows that offsets of a workgroup reach over
        ok &= !p.tiled || ld < (1 << 22);
        ok &= m <= 1 || ((span < m ? span : m) - 1) * 2 * ld + 2 * k <= (int64_t)1 << 31;
        ok &= p.tiled || together <= 16;
        ok &= rows >= 16 || 16 * 2 * ld >= (int64_t)1 << 31;                               // the direct kernel's tokens, where they fit
        ++cases;
        if (!ok && ++bad < 10) std::printf("m=%ld k=%ld ld=%ld: rows=%ld\n", (long)m, (long)k, (long)ld, (long)rows);
    }
    std::printf("cases=%ld bad=%ld\n", cases, bad);
    return bad != 0;
}
