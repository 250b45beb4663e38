// The forms of the layer norm's row kernels: every row takes one that is built and holds its channels, and none is built that no row takes.
#include <cstdio>
#include <set>
#include <tuple>
#include "ftp_norm_rows.h"

using namespace ftp;

int main()
{
    std::set<std::tuple<int, int, bool>> taken;
    for (int vec : {1, 2, 4, 8})
        for (int C = vec; C < 70000; C += vec) {
            const RowForm f = row_form(C, vec);
            if (f.nv == 0) {
                if ((C + vec - 1) / vec <= 256 * row_most(vec)) { std::printf("%d channels in vectors of %d would fit\n", C, vec); return 1; }
                continue;
            }
            if (!row_built(vec, f.nv, f.wide) || (long long)f.lanes * f.nv * vec < C || f.wide != (f.lanes == 256) || (f.lanes & (f.lanes - 1))) {
                std::printf("%d channels in vectors of %d: %d lanes, %d vectors, wide %d\n", C, vec, f.lanes, f.nv, f.wide);
                return 1;
            }
            taken.insert({vec, f.nv, f.wide});
        }
    for (int vec : {1, 2, 4, 8})
        for (int nv : {1, 2, 4, 8})
            for (bool wide : {false, true})
                if (row_built(vec, nv, wide) != (taken.count({vec, nv, wide}) > 0)) {
                    std::printf("vectors of %d, %d a lane, wide %d: %s\n", vec, nv, wide, row_built(vec, nv, wide) ? "built, but nothing takes it" : "taken, but not built");
                    return 1;
                }
    std::printf("ok\n");
    return 0;
}
