/*
 * How group norm cuts up a call, on the CPU: reads lines of
 *   samples positions channels groups dtype gradient
 * and prints for each the kernel variant that it takes: threads, pieces,
 * whether the 8 columns of a thread lie in one group, and whether the
 * positions are cut into chunks.  What the kernels assume of a plan is checked.
 */
#include <cstdio>

#include "groupnorm.hpp"

namespace msvm {

static int run()
{
    long long n, p, ch, g, c;
    int t, grad, bad = 0;
    while (std::scanf("%lld %lld %lld %lld %d %d", &n, &p, &ch, &g, &t,
                      &grad) == 6) {
        const Plan a = plan_of(n, p, ch, g, t, grad != 0);
        std::printf("%d %d %d %d\n", a.threads, a.pieces, (int)a.even,
                    (int)a.split());
        if (!n) continue;
        c = (a.chunk + a.rows - 1) / a.rows;
        const bool fine =
            a.lanes * a.rows <= a.threads && a.rows >= 1 && c <= a.pieces &&
            a.chunk >= 1 && a.chunk * a.chunks >= p && a.cols <= 8 * a.lanes &&
            a.groups <= (a.threads < 256 ? 2 * a.threads : 512) &&
            a.groups * a.slices / a.parts_across >= g &&
            a.pieces <= most_pieces(t, grad != 0) &&
            a.pieces == pieces_of(a.threads, a.pieces) &&
            (a.split() ? a.threads >= 256 && a.pieces <= 8 : true);
        if (!fine) {
            std::fprintf(stderr, "%lld x %lld x %lld in %lld: a plan of %d "
                         "threads, %d pieces\n", n, p, ch, g, a.threads,
                         a.pieces);
            bad = 1;
        }
    }
    return bad;
}

}  // namespace msvm

int main() { return msvm::run(); }
