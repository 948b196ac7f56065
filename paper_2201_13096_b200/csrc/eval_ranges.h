// Index arithmetic of the evaluation operators that the host can check: plain C++, for device code too.
#ifndef SPDY_EVAL_RANGES_H
#define SPDY_EVAL_RANGES_H

#ifdef __CUDACC__
#define SPDY_EVAL_FN __host__ __device__ __forceinline__
#else
#define SPDY_EVAL_FN inline
#endif

#include <stdint.h>

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

// Division of 32-bit numbers by one that the host knows: the upper half of x ceil(2^64 / d), exact for every x.  (With the compiler's
// divisions the places of tiles and shares took 300 instructions a tile and warp, as many as carrying the tile on.)
struct Divisor {
    uint64_t m;
    uint32_t d;
    SPDY_EVAL_FN Divisor(uint32_t by = 1) : m(by > 1 ? ~0ull / by + 1 : 0), d(by) {}
    SPDY_EVAL_FN uint32_t of(uint32_t x) const
    {
        if (d == 1) return x;
#ifdef __CUDA_ARCH__
        return static_cast<uint32_t>(__umul64hi(x, m));
#else
        return static_cast<uint32_t>(static_cast<unsigned __int128>(x) * m >> 64);
#endif
    }
};

// Tiles of a matrix in the order they are worked on: groups of `group` tiles down (the last one may be lower), all tiles across before the
// next group; one such sequence after the other for each share of a sum.
struct Tiles {
    int down, group;
    Divisor all, per_group, per_rows, per_last;  // tiles; of a group; down in a group, in the last one
    SPDY_EVAL_FN Tiles(int m = 1, int n = 1, int most = 1)
        : down(m), group(most < m ? most : m), all(static_cast<uint32_t>(m) * n), per_group(static_cast<uint32_t>(group) * n), per_rows(group),
          per_last(m % group ? m % group : group)
    {
    }
    SPDY_EVAL_FN uint32_t count() const { return all.d; }
    SPDY_EVAL_FN void at(uint32_t item, int &share, int &tm, int &tn) const
    {
        share = static_cast<int>(all.of(item));
        const uint32_t tile = item - static_cast<uint32_t>(share) * all.d, g = per_group.of(tile), rest = tile - g * per_group.d;
        const bool last = static_cast<int>((g + 1) * per_rows.d) > down;
        const uint32_t across = last ? per_last.of(rest) : per_rows.of(rest);
        tn = static_cast<int>(across);
        tm = static_cast<int>(g * per_rows.d + rest - across * (last ? per_last.d : per_rows.d));
    }
};

}  // namespace spdy_eval
#endif
