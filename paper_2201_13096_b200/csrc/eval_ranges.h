// Index arithmetic of the evaluation operators that the host can check: plain C++, for device code too.
#ifndef SPDY_EVAL_RANGES_H
#define SPDY_EVAL_RANGES_H

#ifdef __CUDACC__
#define SPDY_EVAL_FN __host__ __device__ __forceinline__
#else
#define SPDY_EVAL_FN inline
#endif

namespace spdy_eval {

// Whether elements e .. e + n - 1 of a vector of D can be read `granule` at a time: `aligned`, the vector starts on a granule, and
// all of them lie inside (e is negative where a row's first granule begins before the row).
SPDY_EVAL_FN bool in_granules(bool aligned, int e, int n, int D, int granule) { return aligned && n % granule == 0 && e >= 0 && e % granule == 0 && e <= D - n; }

// The patience of a wait that polls, in cycles of a counter that goes on while the kernel is preempted: what passes between two
// polls counts for at most `kMostBetween`, so that only time in which the kernel ran and nothing came uses it up.
struct Patience {
    static constexpr long long kLimit = 4000000000ll, kMostBetween = 1ll << 20;  // two seconds, half a millisecond
    long long last = 0, waited = 0;
    SPDY_EVAL_FN bool over(long long now)
    {
        if (last != 0) waited += now - last < kMostBetween ? now - last : kMostBetween;
        last = now;
        return waited > kLimit;
    }
};

}  // namespace spdy_eval
#endif
