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

}  // namespace spdy_eval
#endif
