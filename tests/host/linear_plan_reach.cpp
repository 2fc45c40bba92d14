// Which kernels the cut of a projection (csrc/linear_plan.hpp) asks for, over the range of sizes: one line each,
// "kind tiled nt mt".
#include <cstdio>
#include <set>
#include <tuple>

#include "../../paper_2605_08565_amd/csrc/linear_plan.hpp"

int main()
{
    std::set<std::tuple<int, int, int, int>> seen;
    for (int m = 1; m <= 50000; m = m < 70 ? m + 1 : m * 3 / 2)
        for (int n : {1, 64, 1024, 4096, 14336, 16384, 16385, 28672, 128000})
            for (int k : {32, 1024, 4096, 14336})
                for (int kind = 0; kind < 3; ++kind)       // bf16, Q8 widened, Q8 as it is
                    for (int rank : {0, 16}) {
                        const mxq::LinearPlan p = mxq::plan_linear({m, n, k, 32, kind == 0, kind == 2, rank});
                        seen.insert({kind, p.tiled, p.nt, p.mt});
                    }
    for (const auto& [kind, tiled, nt, mt] : seen) std::printf("%d %d %d %d\n", kind, tiled, nt, mt);
}
