// apex::rows_overlap against every pair of bytes, over small rows, strides and distances.
#include <cstdio>
#include <vector>

#include "common.h"

int main() {
    static char base[4096];
    const char *middle = base + 2048;
    long checked = 0, overlaps = 0;
    for (int T = 1; T <= 4; ++T)
        for (int an = 1; an <= 4; ++an)
            for (int as = an; as <= an + 3; ++as)
                for (int bn = 1; bn <= 4; ++bn)
                    for (int bs = bn; bs <= bn + 3; ++bs)
                        for (int d = -40; d <= 40; ++d) {
                            bool want = false;
                            for (int i = 0; i < T; ++i)
                                for (int j = 0; j < T; ++j) {
                                    const int a = i * as, b = d + j * bs;
                                    want = want || (a < b + bn && b < a + an);
                                }
                            const bool got = apex::rows_overlap({middle, as, an}, {middle + d, bs, bn}, T);
                            if (got != want) {
                                std::printf("T=%d a %d of %d, b %d of %d, distance %d: %d\n", T, an, as, bn, bs, d, got);
                                return 1;
                            }
                            ++checked, overlaps += want;
                        }
    // rows behind the 2^32nd byte
    const int64_t far = int64_t(1) << 33;
    if (apex::rows_overlap({middle, far, 16}, {middle + 16, far, 16}, 1 << 20) ||
        !apex::rows_overlap({middle, far, 16}, {middle + 8, far, 16}, 1 << 20))
        return 1;
    std::printf("%ld checked, %ld overlap\nok\n", checked, overlaps);
    return 0;
}
