// Which kernels take the products of matrices that are orthogonalised together, for tests on a host without a GPU: reads lines "steps a b c count" and
// `count` times "rows cols copies"; prints "thin rounds", then of every round one character a matrix: the kernel (. none, 0 1 straight from
// the caches, 2 3 through LDS, 4 divided), rounds by spaces.
#include <cstdio>

#include "pex_internal.h"

int main()
{
    int steps, count;
    float a, b, c;
    while (scanf("%d %f %f %f %d", &steps, &a, &b, &c, &count) == 5) {
        pex::NsMatrix m[pex::NS_GROUP] = {};
        for (int i = 0; i < count; ++i) {
            long long rows, cols, copies;
            if (scanf("%lld %lld %lld", &rows, &cols, &copies) != 3) return 1;
            m[i] = {nullptr, nullptr, nullptr, rows, cols, copies, 0.f};
        }
        const pex::NsCall call = {a, b, c, 1e-7f, steps, 0.f, 0.f, 0.f, 0};
        static pex::NsPlan plan;
        pex::plan_newton_schulz(m, count, call, plan);
        printf("%d %d", (int)plan.thin, plan.rounds);
        for (int r = 0; r < plan.rounds; ++r) {
            putchar(' ');
            for (int i = 0; i < count; ++i) putchar(plan.round[r].kernel[i] < 0 ? '.' : '0' + plan.round[r].kernel[i]);
        }
        putchar('\n');
    }
    return 0;
}
