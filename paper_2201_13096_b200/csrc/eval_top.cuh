// The largest elements of a row, for the rows that belong to a block or a cluster (see eval_loss.cuh, which includes this after
// eval_common.cuh).  The file includes nothing itself and reads memory only by way of Row and the loads beside it, so that the host compiler
// can run it too, thread by thread in an order of a test's choice.
#ifndef SPDY_EVAL_TOP_CUH
#define SPDY_EVAL_TOP_CUH

namespace spdy_eval {

// An element's rank is its 64-bit key: the value's bits mapped to an unsigned order above, the complement of the index
// below, so that all keys differ and a larger key is a larger value or an equal one with a lower index.  -0 counts as 0,
// NaN as less than -inf.
__device__ __forceinline__ uint32_t ordered(float x)
{
    if (x != x) return 0u;
    const uint32_t b = __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o)
{
    if (o == 0u) return quiet_nan();
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t index) { return static_cast<uint64_t>(ordered(x)) << 32 | static_cast<uint32_t>(~index); }

// The r-th largest key of a warp's lanes, each lane holding one (0 = none); 0 if fewer than r lanes hold one.
__device__ __forceinline__ uint64_t warp_nth_key(uint32_t value, uint32_t index, int r)
{
    uint64_t last = 0;
    for (int q = 0; q < r; ++q) {
        const uint32_t v = __reduce_max_sync(0xffffffffu, value);
        const uint32_t i = __reduce_min_sync(0xffffffffu, value == v ? index : 0xffffffffu);
        last = static_cast<uint64_t>(v) << 32 | static_cast<uint32_t>(~i);
        if (value == v && index == i) value = 0u, index = 0xffffffffu;
    }
    return last;
}

constexpr int kCandidates = 1536, kListed = 512;

struct TopShared {
    uint64_t cand[kCandidates + 1];  // the last of each takes what is too many
    uint64_t list[kListed + 1];
    uint64_t best[SPDY_TOP_MAX];  // the result, descending
    uint64_t tau[32];
    uint32_t count, count2, entries;  // candidates, block_count's, the list's
    uint32_t hist[256];
    uint64_t prefix;
    uint32_t want;
};

template <int NT> __device__ __forceinline__ int block_count(TopShared &sh, int mine)
{
    mine = __reduce_add_sync(0xffffffffu, mine);
    if (threadIdx.x == 0) sh.count2 = 0;
    __syncthreads();
    if ((threadIdx.x & 31) == 0) atomicAdd(&sh.count2, static_cast<uint32_t>(mine));
    __syncthreads();
    const int total = static_cast<int>(sh.count2);
    __syncthreads();
    return total;
}

// Writes the `want` largest of sh.cand[0..n) in descending order to sh.best (want <= n).  All threads of the block.
template <int NT> __device__ __noinline__ void select_top(TopShared &sh, int n, int want)
{
    uint64_t least = 0;
    if (n > 512) {  // too many to rank all by counting: the want-th largest key first, bit by bit
        for (int b = 63; b >= 0; --b) {
            const uint64_t trial = least | 1ull << b;
            int mine = 0;
            for (int i = threadIdx.x; i < n; i += NT) mine += sh.cand[i] >= trial;
            if (block_count<NT>(sh, mine) >= want) least = trial;
        }
    }
    for (int i = threadIdx.x; i < n; i += NT) {
        const uint64_t k = sh.cand[i];
        if (k < least) continue;
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < n; ++j) rank += sh.cand[j] > k;
        if (rank < want) sh.best[rank] = k;
    }
    __syncthreads();
}

// The `want` largest keys of granules [g0, g1) of a row into sh.cand, by reading the row once per key byte: for rows whose
// order defeats the bound below.  All threads of the block.
template <class T, int NT> __device__ __noinline__ void radix_top(TopShared &sh, const Row<T> row, int g0, int g1, int want)
{
    const int tid = threadIdx.x;
    uint64_t prefix = 0, mask = 0;
    int need = want;
    for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += NT) sh.hist[i] = 0;
        __syncthreads();
        for (int g = g0 + tid; g < g1; g += NT) {
            const int e = row.first(g);
            float f[Elem<T>::kVec];
            Elem<T>::unpack(row.load(g), f);
#pragma unroll
            for (int i = 0; i < Elem<T>::kVec; ++i) {
                if (e + i < 0 || e + i >= row.n) continue;
                const uint64_t k = rank_key(f[i], static_cast<uint32_t>(e + i));
                if ((k & mask) == prefix) atomicAdd(&sh.hist[k >> shift & 255], 1u);
            }
        }
        __syncthreads();
        if (tid == 0) {
            int b = 255, have = 0;
            while (b > 0 && have + static_cast<int>(sh.hist[b]) < need) have += static_cast<int>(sh.hist[b--]);
            sh.prefix = prefix | static_cast<uint64_t>(b) << shift;
            sh.want = static_cast<uint32_t>(need - have);
        }
        __syncthreads();
        prefix = sh.prefix;
        need = static_cast<int>(sh.want);
        mask |= 255ull << shift;
        __syncthreads();
    }
    if (tid == 0) sh.count = 0;
    __syncthreads();
    for (int g = g0 + tid; g < g1; g += NT) {
        const int e = row.first(g);
        float f[Elem<T>::kVec];
        Elem<T>::unpack(row.load(g), f);
#pragma unroll
        for (int i = 0; i < Elem<T>::kVec; ++i) {
            if (e + i < 0 || e + i >= row.n) continue;
            const uint64_t k = rank_key(f[i], static_cast<uint32_t>(e + i));
            if (k >= prefix) {
                const uint32_t at = atomicAdd(&sh.count, 1u);
                if (at < static_cast<uint32_t>(want)) sh.cand[at] = k;
            }
        }
    }
    __syncthreads();
}

// Appends granule g's elements of at least `least` to the candidates.
template <class T> __device__ __noinline__ void append_candidates(TopShared &sh, const T *p, int n, int lead, int g, uint32_t least)
{
    const int e = g * Elem<T>::kVec - lead;
    float f[Elem<T>::kVec];
    Elem<T>::unpack(e >= 0 && e <= n - Elem<T>::kVec ? load_stream(p + e) : load_part(p, n, e), f);
#pragma unroll
    for (int j = 0; j < Elem<T>::kVec; ++j) {
        if (ordered(f[j]) < least || e + j < 0 || e + j >= n) continue;
        sh.cand[min(atomicAdd(&sh.count, 1u), static_cast<uint32_t>(kCandidates))] = rank_key(f[j], static_cast<uint32_t>(e + j));
    }
}

// While a block streams its part of a row, each thread notes the largest element of each of its groups (the U granules of
// one step, or of 2^shift steps in a row too long for the list), NaN for a group without elements.
// Then the K-th largest group value v bounds the K-th largest element from below: elements above v lie in fewer than K
// groups, which are read again; what may still be missing are elements equal to v, those with the lowest ids.
// Result in sh.best[0..want).
template <class T, int NT, int U>
__device__ __forceinline__ void find_top(TopShared &sh, const float *largest, int n_groups, int shift, const Row<T> row, int g0, int g1, int want)
{
    constexpr int NW = NT / 32, STEP = NT * U, VEC = Elem<T>::kVec;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const auto group = [&](int i) { return ordered(largest[i]); };
    // a cheap bound first: the r-th largest lane of every warp, r such that the warps together have `want` lanes above it
    uint32_t lane_best = 0;
    for (int i = 0; i < n_groups; ++i) lane_best = max(lane_best, group(i * NT + tid));
    const uint64_t mine = warp_nth_key(lane_best, static_cast<uint32_t>(lane), (want + NW - 1) / NW);
    if (lane == 0) sh.tau[warp] = mine >> 32;
    if (tid == 0) sh.count = sh.entries = sh.want = 0;
    __syncthreads();
    const uint32_t tau = max(1u, __reduce_min_sync(0xffffffffu, lane < NW ? static_cast<uint32_t>(sh.tau[lane]) : 0xffffffffu));
    const int total = n_groups * NT;
#pragma unroll 4
    for (int i = tid; i < total; i += NT)
        if (group(i) >= tau) {
            sh.list[min(atomicAdd(&sh.entries, 1u), static_cast<uint32_t>(kListed))] = static_cast<uint64_t>(group(i)) << 32 | static_cast<uint32_t>(~i);
        }
    __syncthreads();
    int listed = static_cast<int>(sh.entries);  // decides which way all threads take: never written again
    const int each = U << shift;
    if (listed <= kListed && listed >= want) {
        // the common case: every group that can hold one of the best is listed, those equal to v among them
        for (int i = tid; i < listed; i += NT) {
            const uint64_t k = sh.list[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < listed; ++j) rank += sh.list[j] > k;
            if (rank == want - 1) sh.want = static_cast<uint32_t>(k >> 32);
        }
        __syncthreads();
        const uint32_t least = sh.want;
        for (int i = tid; i < listed * each; i += NT) {
            const uint64_t k = sh.list[i / each];
            if (static_cast<uint32_t>(k >> 32) < least) continue;
            const int slot = static_cast<int>(~static_cast<uint32_t>(k));
            const int g = g0 + (slot / NT << shift) * STEP + slot % NT + i % each * NT;
            if (g >= g1) continue;
            append_candidates<T>(sh, row.p, row.n, row.lead, g, least);
        }
        __syncthreads();
        int have = static_cast<int>(sh.count);
        if (have > kCandidates || have < want) {
            __syncthreads();
            radix_top<T, NT>(sh, row, g0, g1, want);
            have = want;
        }
        select_top<NT>(sh, have, want);
        return;
    }
    uint32_t v = 0;  // stays 0 with fewer groups than `want`: every element is looked at
    if (listed > kListed) {
        for (int b = 31; b >= 0; --b) {
            const uint32_t trial = v | 1u << b;
            int count = 0;
            for (int i = tid; i < total; i += NT) count += group(i) >= trial;
            if (block_count<NT>(sh, count) >= want) v = trial;
        }
    }
    // the groups that can hold one of the best: those above v, and those equal to v unless they are many
    int ties = 0, above = 0;
    for (int i = tid; i < total; i += NT) ties += group(i) == v, above += group(i) > v;
    ties = block_count<NT>(sh, ties);
    above = block_count<NT>(sh, above);
    const bool few = ties + above <= kListed && ties <= 64 + want;
    const uint32_t least = few ? v : v + 1;
    if (tid == 0) sh.count = sh.count2 = 0;
    __syncthreads();
    for (int i = tid; i < total; i += NT)
        if (group(i) >= least) sh.list[atomicAdd(&sh.count2, 1u)] = i;
    __syncthreads();
    listed = static_cast<int>(sh.count2);
    for (int i = tid; i < listed * each; i += NT) {
        const int slot = static_cast<int>(sh.list[i / each]);
        const int g = g0 + (slot / NT << shift) * STEP + slot % NT + i % each * NT;
        if (g >= g1) continue;
        append_candidates<T>(sh, row.p, row.n, row.lead, g, least);
    }
    __syncthreads();
    int have = static_cast<int>(sh.count);
    __syncthreads();
    if (!few && have < want) {
        // many groups equal to v (a masked or constant row): its elements in ascending order until there are enough
        for (int base = g0; base < g1 && have < want; base += NT) {
            const int g = base + tid;
            uint32_t bits = 0;
            float f[VEC];
            const int e = row.first(g);
            if (g < g1) {
                Elem<T>::unpack(row.load(g), f);
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (ordered(f[j]) == v && e + j >= 0 && e + j < row.n) bits |= 1u << j;
            }
            int before = __popc(bits);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int other = __shfl_up_sync(0xffffffffu, before, d);
                if (lane >= d) before += other;
            }
            if (lane == 31) sh.tau[warp] = before;
            __syncthreads();
            int total_here = 0;
            for (int w = 0; w < NW; ++w) {
                if (w == warp) before += total_here;
                total_here += static_cast<int>(sh.tau[w]);
            }
            int at = have + before - __popc(bits);
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (bits >> j & 1) {
                    if (at < want) sh.cand[at] = rank_key(f[j], static_cast<uint32_t>(e + j));
                    ++at;
                }
            have += total_here;
            __syncthreads();
        }
        have = min(have, want);
    }
    if (have > kCandidates || have < want) {
        radix_top<T, NT>(sh, row, g0, g1, want);
        have = want;
    }
    select_top<NT>(sh, have, want);
}

}  // namespace spdy_eval
#endif
