// What the kernels read in granules lies inside (csrc/eval_ranges.h).
#include <stdio.h>

#include <initializer_list>

#include "../../paper_2201_13096_b200/csrc/eval_ranges.h"

int main()
{
    int failures = 0;
    for (int D = 1; D <= 80; ++D)
        for (int granule : {4, 8})
            for (int n : {1, 4, 8})
                for (int e = -8; e <= D + 8; ++e) {
                    const bool inside = e >= 0 && e + n <= D, whole = n % granule == 0 && e % granule == 0;
                    if (spdy_eval::in_granules(true, e, n, D, granule) != (inside && whole) || spdy_eval::in_granules(false, e, n, D, granule)) {
                        if (++failures <= 10) printf("%d elements from %d on of %d in granules of %d: %s\n", n, e, D, granule, inside ? "inside" : "out of range");
                    }
                }
    return failures != 0;
}
