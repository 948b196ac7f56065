// What the kernels read in granules lies inside, and waits give up neither too early nor never (csrc/eval_ranges.h).
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
    const long long limit = spdy_eval::Patience::kLimit;
    for (long long between : {100ll, 10000ll, 1ll << 20, 1ll << 30}) {
        // polled steadily: as many polls as fit the limit, each counted for half a millisecond at most
        spdy_eval::Patience patience;
        const long long counted = between < (1ll << 20) ? between : 1ll << 20;
        long long polls = 1, now = 123456789;
        while (!patience.over(now) && polls < (1ll << 27)) ++polls, now += between;
        if (polls != limit / counted + 2) ++failures, printf("gave up after %lld polls every %lld cycles\n", polls, between);
    }
    spdy_eval::Patience preempted;
    long long now = 5;
    for (int k = 0; k < 1000; ++k, now += 1000) {
        if (k == 500) now += 100 * limit;  // others had the device for minutes
        if (preempted.over(now)) {
            ++failures;
            printf("gave up for time in which the kernel did not run\n");
            break;
        }
    }
    return failures != 0;
}
