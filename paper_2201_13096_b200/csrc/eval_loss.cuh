// Kernels over rows of logits: log probabilities of given tokens (with entropy and top alternatives), the distillation
// loss, and their gradients.  Instantiated in eval_token_logprobs.cu and eval_distill.cu.
//
// Mathematics.  Everything is kept in base 2: with c = log2(e) / T and the running maximum m of the logits, d_v = (x_v - m) c
// and s = sum 2^d, a probability is 2^d_v / s.  The difference is taken before the scaling: for 16-bit logits it is exact,
// and rows of the type's lowest value do not overflow.  The entropy needs t = sum 2^d d beside s: H = ln 2 (log2 s - t / s).
// When the maximum rises by delta / c, s becomes s 2^-delta and t becomes (t - s delta) 2^-delta.
// An element costs half an instruction each for difference, scaling and sum (two to an instruction), one to unpack and one
// for the special-function unit, whose 16 results a cycle and multiprocessor are the next limit behind memory.
#ifndef SPDY_EVAL_LOSS_CUH
#define SPDY_EVAL_LOSS_CUH

#include <type_traits>

#include "eval_common.cuh"

namespace spdy_eval {

namespace cg = cooperative_groups;

struct LossArgs {
    const void *logits;
    int64_t ld, R, V;
    float c, inv_t, temperature;  // c = log2(e) / T
    const void *ids;         // tokens [R] or the teacher's ids [R][K]
    int index_bits;
    int32_t K;               // top_k or the teacher's entries
    const float *top_lp;     // teacher's log probabilities [R][K]
    // results
    float *logprob, *entropy, *lse, *loss, *rest;
    int32_t *top_ids;
    float *top_logprobs;
    // backward
    const float *in_lse, *in_entropy, *in_rest, *grad, *grad_entropy;
    void *dlogits;
    int64_t lddl;
    int segments;            // blocks per row of the backward kernel
};

__device__ __forceinline__ int64_t index_at(const void *ids, int bits, int64_t i)
{
    return bits == 64 ? static_cast<const int64_t *>(ids)[i] : static_cast<int64_t>(static_cast<const int32_t *>(ids)[i]);
}

// A row's token: -1 for none, V for any id beyond the vocabulary.
__device__ __forceinline__ int token_at(const LossArgs &a, int64_t r)
{
    const int64_t t = index_at(a.ids, a.index_bits, r);
    return t < 0 ? -1 : static_cast<int>(t < a.V ? t : a.V);
}

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    return x;
}
__device__ __forceinline__ float warp_max(float x)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}

// Softmax sums of a warp, block or cluster.
struct Stats {
    float m, s, t;  // sums over everything (or, with a teacher's tail, over what lies outside its set; t: entropy only)
    float mi, si;   // sums over the teacher's set
};

__device__ __forceinline__ void join_entropy(float &m, float &s, float &t, float om, float os, float ot, float c)
{
    const float top = fmaxf(m, om);
    float s2 = 0.f, t2 = 0.f;
    if (s != 0.f) {
        const float d = max_nan((m - top) * c, -1000.f), f = ex2(d);
        s2 = s * f;
        t2 = f * fmaf(s, d, t);
    }
    if (os != 0.f) {
        const float d = max_nan((om - top) * c, -1000.f), f = ex2(d);
        s2 = fmaf(os, f, s2);
        t2 = fmaf(f, fmaf(os, d, ot), t2);
    }
    m = top, s = s2, t = t2;
}

template <bool ENT, bool TAIL> __device__ __forceinline__ void join_stats(Stats &a, const Stats &b, float c)
{
    if (ENT) join_entropy(a.m, a.s, a.t, b.m, b.s, b.t, c);
    else join_sums(a.m, a.s, b.m, b.s, c);
    if (TAIL) join_sums(a.mi, a.si, b.mi, b.si, c);
}

template <bool ENT, bool TAIL> __device__ __forceinline__ Stats shuffle_xor(const Stats &a, int d)
{
    Stats b = {};
    b.m = __shfl_xor_sync(0xffffffffu, a.m, d);
    b.s = __shfl_xor_sync(0xffffffffu, a.s, d);
    if (ENT) b.t = __shfl_xor_sync(0xffffffffu, a.t, d);
    if (TAIL) b.mi = __shfl_xor_sync(0xffffffffu, a.mi, d), b.si = __shfl_xor_sync(0xffffffffu, a.si, d);
    return b;
}

// What a thread has added up: s and t in two halves, even and odd elements.
struct Running {
    float m;
    float2 s, t;
};

// Makes `top` the maximum the sums are relative to, if it is larger.
template <bool ENT> __device__ __forceinline__ void raise(Running &st, float top, float c)
{
    if (top > st.m) {
        if (st.s.x + st.s.y != 0.f) {
            const float d = max_nan((st.m - top) * c, -1000.f), f = ex2(d);
            if (ENT) st.t = mul2(both(f), fma2(st.s, both(d), st.t));
            st.s = mul2(st.s, both(f));
        }
        st.m = top;
    }
}

// Adds a granule; no element is larger than the maximum.
template <class T, bool ENT> __device__ __forceinline__ void accumulate(uint4 raw, float c, Running &st)
{
    const float2 minus = both(st.m == neg_inf() ? 0.f : -st.m), scale = both(c);
    float2 f[Elem<T>::kVec / 2];
    Elem<T>::pairs(raw, f);
#pragma unroll
    for (int i = 0; i < Elem<T>::kVec / 2; ++i) {
        float2 d = mul2(add2(f[i], minus), scale);
        if (ENT) d = make_float2(max_nan(d.x, -1000.f), max_nan(d.y, -1000.f));  // an id that is not allowed adds 0 rather than 0 times -inf
        const float2 e = make_float2(ex2(d.x), ex2(d.y));
        st.s = add2(st.s, e);
        if (ENT) st.t = fma2(e, d, st.t);
    }
}

// -inf in place of the elements whose bit is set
template <class T> __device__ __forceinline__ uint4 without(uint4 raw, uint32_t bits)
{
    float f[Elem<T>::kVec];
    Elem<T>::unpack(raw, f);
#pragma unroll
    for (int i = 0; i < Elem<T>::kVec; ++i)
        if (bits >> i & 1) f[i] = neg_inf();
    return Elem<T>::pack(f);
}

// The bits of granule g (counted from the first one the bitmap covers).
template <class T> __device__ __forceinline__ uint32_t bits_of(const uint32_t *bitmap, int g)
{
    if (Elem<T>::kVec == 8) return reinterpret_cast<const uint8_t *>(bitmap)[g];
    return reinterpret_cast<const uint8_t *>(bitmap)[g >> 1] >> ((g & 1) * 4) & 15u;
}

// ------------------------------------------------------------------------------------------ top alternatives
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

constexpr int kCandidates = 2048;

struct TopShared {
    uint64_t cand[kCandidates];
    uint64_t best[SPDY_TOP_MAX];  // the result, descending
    uint64_t tau[32];
    uint32_t count, count2;
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
        for (int j = 0; j < n; ++j) rank += sh.cand[j] > k;
        if (rank < want) sh.best[rank] = k;
    }
    __syncthreads();
}

// The `want` largest keys of granules [g0, g1) of a row into sh.cand, by reading the row once per key byte: for rows whose
// order defeats the bound below.  All threads of the block.
template <class T, int NT> __device__ __noinline__ void radix_top(TopShared &sh, const Row<T> &row, int g0, int g1, int want)
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

// While a block streams its part of a row, each thread notes the largest element of each of its groups (the U granules of
// one step, or of 2^shift steps in a row too long for `groups`) as an ordered 32-bit value, 0 for a group without elements.
// Then the K-th largest group value v bounds the K-th largest element from below: elements above v lie in fewer than K
// groups, which are read again; what is still missing are elements equal to v, those with the lowest ids.
// `lane_best` is the thread's largest value over all its groups.  Result in sh.best[0..want).
template <class T, int NT, int U>
__device__ __noinline__ void find_top(TopShared &sh, const uint32_t *groups, int n_groups, int shift, uint32_t lane_best, const Row<T> &row, int g0, int g1, int want)
{
    constexpr int NW = NT / 32, STEP = NT * U;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // a cheap bound first: the r-th largest lane of every warp, r such that the warps together have `want` lanes above it
    const uint64_t mine = warp_nth_key(lane_best, static_cast<uint32_t>(lane), (want + NW - 1) / NW);
    if (lane == 0) sh.tau[warp] = mine >> 32;
    if (tid == 0) sh.count = 0;
    __syncthreads();
    const uint32_t tau = max(1u, __reduce_min_sync(0xffffffffu, lane < NW ? static_cast<uint32_t>(sh.tau[lane]) : 0xffffffffu));
    const int total = n_groups * NT;
    for (int i = tid; i < total; i += NT)
        if (groups[i] >= tau) {
            const uint32_t at = atomicAdd(&sh.count, 1u);
            if (at < 512) sh.cand[at] = static_cast<uint64_t>(groups[i]) << 32 | static_cast<uint32_t>(~i);
        }
    __syncthreads();
    const int listed = static_cast<int>(sh.count);
    uint32_t v = 0;
    if (listed > 512) {
        for (int b = 31; b >= 0; --b) {
            const uint32_t trial = v | 1u << b;
            int count = 0;
            for (int i = tid; i < total; i += NT) count += groups[i] >= trial;
            if (block_count<NT>(sh, count) >= want) v = trial;
        }
    } else {
        if (tid == 0) sh.want = 0;  // fewer groups than `want`: every element is wanted or nearly
        __syncthreads();
        for (int i = tid; i < listed; i += NT) {
            const uint64_t k = sh.cand[i];
            int rank = 0;
            for (int j = 0; j < listed; ++j) rank += sh.cand[j] > k;
            if (rank == want - 1) sh.want = static_cast<uint32_t>(k >> 32);
        }
        __syncthreads();
        v = sh.want;
    }
    __syncthreads();
    if (tid == 0) sh.count = 0;
    __syncthreads();
    // elements above v, and the number of groups whose largest is v
    int ties = 0;
    for (int i = tid; i < total; i += NT) {
        if (groups[i] < v) continue;
        ties += groups[i] == v;
        if (groups[i] == v) continue;
        const int base = g0 + (i / NT << shift) * STEP + i % NT;
        for (int k = 0; k < (U << shift); ++k) {
            const int g = base + k * NT;
            if (g >= g1) break;
            const int e = row.first(g);
            float f[Elem<T>::kVec];
            Elem<T>::unpack(row.load(g), f);
#pragma unroll
            for (int j = 0; j < Elem<T>::kVec; ++j) {
                if (ordered(f[j]) <= v || e + j < 0 || e + j >= row.n) continue;
                const uint32_t at = atomicAdd(&sh.count, 1u);
                if (at < kCandidates) sh.cand[at] = rank_key(f[j], static_cast<uint32_t>(e + j));
            }
        }
    }
    ties = block_count<NT>(sh, ties);
    const int above = static_cast<int>(sh.count);
    __syncthreads();
    if (above < want && ties <= 64) {
        // few groups can hold an element equal to v: take them all
        for (int i = tid; i < total; i += NT) {
            if (groups[i] < v) continue;
            const int base = g0 + (i / NT << shift) * STEP + i % NT;
            for (int k = 0; k < (U << shift); ++k) {
                const int g = base + k * NT;
                if (g >= g1) break;
                const int e = row.first(g);
                float f[Elem<T>::kVec];
                Elem<T>::unpack(row.load(g), f);
#pragma unroll
                for (int j = 0; j < Elem<T>::kVec; ++j) {
                    if (ordered(f[j]) != v || e + j < 0 || e + j >= row.n) continue;
                    const uint32_t at = atomicAdd(&sh.count, 1u);
                    if (at < kCandidates) sh.cand[at] = rank_key(f[j], static_cast<uint32_t>(e + j));
                }
            }
        }
        __syncthreads();
    } else if (above < want) {
        // many (a masked or constant row): in ascending order from the row's start until there are enough
        int have = above;
        for (int base = g0; base < g1 && have < want; base += NT) {
            const int g = base + tid;
            uint32_t bits = 0;
            float f[Elem<T>::kVec];
            const int e = row.first(g);
            if (g < g1) {
                Elem<T>::unpack(row.load(g), f);
#pragma unroll
                for (int j = 0; j < Elem<T>::kVec; ++j)
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
            for (int j = 0; j < Elem<T>::kVec; ++j)
                if (bits >> j & 1) {
                    if (at < want) sh.cand[at] = rank_key(f[j], static_cast<uint32_t>(e + j));
                    ++at;
                }
            have += total_here;
            __syncthreads();
        }
        if (tid == 0) sh.count = static_cast<uint32_t>(min(have, want));
        __syncthreads();
    }
    int n = static_cast<int>(sh.count);
    __syncthreads();
    if (n > kCandidates || n < want) {
        radix_top<T, NT>(sh, row, g0, g1, want);
        n = want;
    }
    select_top<NT>(sh, n, want);
}

// ------------------------------------------------------------------------------------------ teacher's entries
struct TeacherShared {
    int32_t id[SPDY_DISTILL_MAX];  // -1: no entry
    float q[SPDY_DISTILL_MAX], logq[SPDY_DISTILL_MAX];
    float x[SPDY_DISTILL_MAX];     // the student's logit at id
    float left, mass;              // mass: sum of q
    int bad;                       // an id >= V
};

// The entries of a row; the student's logits only for ids in [e0, e1) (another block may be overwriting the rest in place).
template <class T, int NT> __device__ __forceinline__ void teacher_read(TeacherShared &sh, const LossArgs &a, int64_t row, int64_t e0, int64_t e1)
{
    if (threadIdx.x == 0) sh.bad = 0;
    __syncthreads();
    for (int j = threadIdx.x; j < a.K; j += NT) {
        const int64_t id = index_at(a.ids, a.index_bits, row * a.K + j);
        if (id >= a.V) sh.bad = 1;
        const bool here = id >= 0 && id < a.V;
        sh.id[j] = here ? static_cast<int32_t>(id) : -1;
        sh.logq[j] = here ? a.top_lp[row * a.K + j] : neg_inf();
        sh.x[j] = here && id >= e0 && id < e1 ? Elem<T>::to_float(static_cast<const T *>(a.logits)[row * a.ld + id]) : neg_inf();
    }
}

// q, log q, left and mass from the entries; one warp, after a barrier behind teacher_read.
template <bool TAIL> __device__ __forceinline__ void teacher_weights(TeacherShared &sh, int K)
{
    const int lane = threadIdx.x & 31;
    float sum = 0.f;
    if (TAIL) {
        for (int j = lane; j < K; j += 32) {
            sh.q[j] = expf(sh.logq[j]);
            sum += sh.q[j];
        }
        sum = warp_sum(sum);
        if (lane == 0) sh.left = sum < 1.f ? 1.f - sum : 0.f, sh.mass = sum;
    } else {
        float top = neg_inf();
        for (int j = lane; j < K; j += 32) top = fmaxf(top, sh.logq[j]);
        top = warp_max(top);
        const float base = top == neg_inf() ? 0.f : top;
        for (int j = lane; j < K; j += 32) {
            sh.q[j] = expf(sh.logq[j] - base);
            sum += sh.q[j];
        }
        sum = warp_sum(sum);
        const float log_sum = logf(sum);
        for (int j = lane; j < K; j += 32) {
            sh.q[j] = sum == 0.f ? 0.f : sh.q[j] / sum;
            sh.logq[j] = sum == 0.f ? neg_inf() : sh.logq[j] - base - log_sum;
        }
        if (lane == 0) sh.left = 0.f, sh.mass = sum == 0.f ? 0.f : sum / sum;
    }
    __syncwarp();
}

// What a row's losses and gradients need of the sums.
struct RowEnd {
    float m, s, ls;    // all: maximum, the sum relative to it and its log2
    float mr, sr, lsr; // outside the teacher's set
    bool empty, rest_empty;
};

template <bool TAIL> __device__ __forceinline__ RowEnd row_end(const Stats &st, float c)
{
    RowEnd e;
    e.mr = st.m, e.sr = st.s, e.lsr = log2f(st.s), e.rest_empty = st.s == 0.f;
    float m = st.m, s = st.s;
    if (TAIL) join_sums(m, s, st.mi, st.si, c);
    e.m = m, e.s = s, e.ls = log2f(s), e.empty = s == 0.f;
    return e;
}
__device__ __forceinline__ float lse_of(float m, float ls, bool empty, float inv_t) { return empty ? neg_inf() : fmaf(m, inv_t, kLn2 * ls); }
__device__ __forceinline__ float log_prob(float x, const RowEnd &e, float inv_t) { return e.empty ? neg_inf() : fmaf(x - e.m, inv_t, -kLn2 * e.ls); }

// One warp: the loss of a row, in all lanes.
template <bool TAIL> __device__ __forceinline__ float teacher_loss(const TeacherShared &sh, const RowEnd &e, float inv_t, int K)
{
    const int lane = threadIdx.x & 31;
    float sum = 0.f;
    for (int j = lane; j < K; j += 32) {
        const float q = sh.q[j];
        if (q == 0.f) continue;
        sum += q * (sh.logq[j] - log_prob(sh.x[j], e, inv_t));
    }
    sum = warp_sum(sum);
    if (TAIL && !e.rest_empty && !(sh.left == 0.f)) sum += sh.left * (logf(sh.left) - fmaf(e.mr - e.m, inv_t, kLn2 * (e.lsr - e.ls)));
    return sh.bad ? quiet_nan() : sum;
}

// ------------------------------------------------------------------------------------------ forward
enum { kLogprobs = 0, kLogprobsTop = 1, kDistill = 2, kDistillTail = 3 };

constexpr int kBitmapWords = 4096;  // ids of one segment of a row: 2^17 bits
constexpr int kGroupSteps = 32;     // groups a thread notes at most

template <int NT> struct ForwardShared {
    Stats part[NT / 32];
    Stats pub;           // this block's sums, read by the cluster's first block
    uint32_t found;      // entries of top.best
};

// Sums of a warp's threads, then of the block's warps (in warp 0 afterwards).
template <bool ENT, bool TAIL, int NT> __device__ __forceinline__ Stats block_stats(const Running &run, float mi, float si, Stats *part, float c)
{
    constexpr int NW = NT / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // the warp's maximum first, so that every lane rescales once and the rest are additions
    Stats st = {warp_max(run.m), run.s.x + run.s.y, ENT ? run.t.x + run.t.y : 0.f, mi, si};
    if (st.s != 0.f) {
        const float d = max_nan((run.m - st.m) * c, -1000.f), f = ex2(d);
        if (ENT) st.t = f * fmaf(st.s, d, st.t);
        st.s *= f;
    }
    st.s = warp_sum(st.s);
    if (ENT) st.t = warp_sum(st.t);
    if (TAIL) {
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const float om = __shfl_xor_sync(0xffffffffu, st.mi, d), os = __shfl_xor_sync(0xffffffffu, st.si, d);
            join_sums(st.mi, st.si, om, os, c);
        }
    }
    if (lane == 0) part[warp] = st;
    __syncthreads();
    if (warp == 0) {
        st = lane < NW ? part[lane] : Stats{neg_inf(), 0.f, 0.f, neg_inf(), 0.f};
#pragma unroll
        for (int d = NW / 2; d; d >>= 1) join_stats<ENT, TAIL>(st, shuffle_xor<ENT, TAIL>(st, d), c);
    }
    return st;
}

// One row per cluster of blocks (of one block when there are rows enough), the row's granules divided among the blocks and
// read once, the next U granules of a thread in flight while the present ones are added up.
template <class T, int NT, int U, int MODE>
__global__ void __launch_bounds__(NT, 768 / NT) loss_forward_kernel(const LossArgs a)
{
    constexpr bool ENT = MODE == kLogprobs || MODE == kLogprobsTop, TOP = MODE == kLogprobsTop;
    constexpr bool TEACHER = MODE >= kDistill, TAIL = MODE == kDistillTail;
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ ForwardShared<NT> sh;
    TopShared &top = *reinterpret_cast<TopShared *>(dynamic);                               // TOP
    uint32_t *groups = reinterpret_cast<uint32_t *>(dynamic + sizeof(TopShared));           // TOP
    TeacherShared &teacher = *reinterpret_cast<TeacherShared *>(dynamic);                   // TEACHER
    uint32_t *bitmap = reinterpret_cast<uint32_t *>(dynamic + sizeof(TeacherShared));       // TAIL

    cg::cluster_group cluster = cg::this_cluster();
    const int C = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int64_t r = blockIdx.x / C;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Row<T> row(static_cast<const T *>(a.logits) + r * a.ld, a.V);
    const int G = row.granules(), per = (G + C - 1) / C;
    const int g0 = min(G, rank * per), g1 = min(G, g0 + per);

    Running run = {neg_inf(), both(0.f), both(0.f)};
    float mi = neg_inf(), si = 0.f;
    uint4 next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = row.load_below(g0 + u * NT + tid, g1);
    if (TEACHER) {
        teacher_read<T, NT>(teacher, a, r, rank == 0 ? 0 : row.first(g0), rank == 0 ? a.V : row.first(g1));
        if (TAIL) {
            const int words = min(kBitmapWords, ((g1 - g0) * Elem<T>::kVec + 31) / 32);
            for (int i = tid; i < words; i += NT) bitmap[i] = 0;
        }
        __syncthreads();
        if (warp == 0 && rank == 0) teacher_weights<TAIL>(teacher, a.K);
    }

    constexpr int kSegment = kBitmapWords * 32 / Elem<T>::kVec;  // granules
    static_assert(kSegment % (NT * U) == 0, "a segment is whole steps");
    const int steps = (g1 - g0 + NT * U - 1) / (NT * U);
    int shift = 0;
    if (TOP)
        while (steps >> shift >= kGroupSteps) ++shift;
    int step = 0;
    uint32_t lane_best = 0;

    for (int seg = g0; seg < g1; seg = TAIL ? seg + kSegment : g1) {
        const int seg_end = TAIL ? min(g1, seg + kSegment) : g1;
        if (TAIL) {  // mark the set's ids; the thread that marks one adds it to the sums over the set
            for (int j = tid; j < a.K; j += NT) {
                const int pos = teacher.id[j] - row.first(seg);
                if (teacher.id[j] >= 0 && pos >= 0 && pos < (seg_end - seg) * Elem<T>::kVec) {
                    const uint32_t bit = 1u << (pos & 31);
                    if (!(atomicOr(&bitmap[pos >> 5], bit) & bit)) add_logit(mi, si, teacher.x[j], a.c);
                }
            }
            __syncthreads();
        }
        for (int base = seg; base < seg_end; base += NT * U, ++step) {
            uint4 cur[U];
#pragma unroll
            for (int u = 0; u < U; ++u) cur[u] = next[u];
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = row.load_below(base + NT * U + u * NT + tid, g1);
            if (TAIL) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int g = base + u * NT + tid;
                    const uint32_t bits = g < seg_end ? bits_of<T>(bitmap, g - seg) : 0u;
                    if (bits) cur[u] = without<T>(cur[u], bits);
                }
            }
            float all = Elem<T>::max_of(cur[0]);
#pragma unroll
            for (int u = 1; u < U; ++u) all = fmaxf(all, Elem<T>::max_of(cur[u]));
            if (TOP) {
                uint32_t key = base + tid < g1 ? ordered(all) : 0u;
                lane_best = max(lane_best, key);
                uint32_t *slot = groups + (step >> shift) * NT + tid;
                if (step & ((1 << shift) - 1)) key = max(key, *slot);
                *slot = key;
            }
            raise<ENT>(run, all, a.c);
#pragma unroll
            for (int u = 0; u < U; ++u) accumulate<T, ENT>(cur[u], a.c, run);
        }
        if (TAIL) {
            __syncthreads();
            for (int j = tid; j < a.K; j += NT) {
                const int pos = teacher.id[j] - row.first(seg);
                if (teacher.id[j] >= 0 && pos >= 0 && pos < (seg_end - seg) * Elem<T>::kVec) bitmap[pos >> 5] = 0;
            }
            __syncthreads();
        }
    }

    Stats st = block_stats<ENT, TAIL, NT>(run, mi, si, sh.part, a.c);
    if (tid == 0) sh.pub = st;
    if (TOP) {
        const int e0 = max(0, row.first(g0)), e1 = min(row.n, row.first(g1));
        const int want = max(0, min(a.K, e1 - e0));
        if (want > 0) find_top<T, NT, U>(top, groups, (steps + (1 << shift) - 1) >> shift, shift, lane_best, row, g0, g1, want);
        if (tid == 0) sh.found = static_cast<uint32_t>(want);
    }
    if (C > 1) {
        cluster.sync();
        if (rank == 0) {
            if (warp == 0) {
                st = lane < C ? *cluster.map_shared_rank(&sh.pub, lane) : Stats{neg_inf(), 0.f, 0.f, neg_inf(), 0.f};
#pragma unroll
                for (int d = 4; d; d >>= 1) join_stats<ENT, TAIL>(st, shuffle_xor<ENT, TAIL>(st, d), a.c);
            }
            if (TOP) {
                int n = 0;  // the blocks' lists side by side
                for (int b = 0; b < C; ++b) {
                    const int m = static_cast<int>(*cluster.map_shared_rank(&sh.found, b));
                    const TopShared *other = cluster.map_shared_rank(&top, b);
                    for (int i = tid; i < m; i += NT) top.cand[n + i] = other->best[i];
                    n += m;
                }
                __syncthreads();
                select_top<NT>(top, n, a.K);
            }
        }
        cluster.sync();  // no block leaves while its shared memory is read
        if (rank != 0) return;
        if (tid == 0) sh.pub = st;
    }
    __syncthreads();
    st = sh.pub;
    const RowEnd e = row_end<TAIL>(st, a.c);
    if (tid == 0) {
        if (a.lse) a.lse[r] = lse_of(e.m, e.ls, e.empty, a.inv_t);
        if (ENT) {
            if (a.entropy) a.entropy[r] = e.empty ? 0.f : kLn2 * (e.ls - st.t / st.s);
            if (a.logprob) {
                const int token = token_at(a, r);
                float lp = 0.f;
                if (token >= a.V) lp = quiet_nan();
                else if (token >= 0) lp = log_prob(Elem<T>::to_float(row.p[token]), e, a.inv_t);
                a.logprob[r] = lp;
            }
        }
        if (TAIL && a.rest) a.rest[r] = lse_of(e.mr, e.lsr, e.rest_empty, a.inv_t);
    }
    if (TEACHER && warp == 0 && a.loss) {
        const float loss = teacher_loss<TAIL>(teacher, e, a.inv_t, a.K);
        if (lane == 0) a.loss[r] = loss;
    }
    if (TOP) {
        for (int i = tid; i < a.K; i += NT) {
            const uint64_t k = top.best[i];
            a.top_ids[r * a.K + i] = static_cast<int32_t>(~static_cast<uint32_t>(k));
            a.top_logprobs[r * a.K + i] = log_prob(unordered(static_cast<uint32_t>(k >> 32)), e, a.inv_t);
        }
    }
}

// ------------------------------------------------------------------------------------------ gradients
// A row's gradient is 2^d (k0 + k1 d) per element with d = (x - m) c, plus a few elements that get their own value.
struct RowGrad {
    float m, k0, k1;
};

template <class T, bool ENT> __device__ __forceinline__ uint4 gradient_of(uint4 raw, float c, const RowGrad &k)
{
    const float2 minus = both(-k.m), scale = both(c), k0 = both(k.k0), k1 = both(k.k1);
    float2 f[Elem<T>::kVec / 2];
    Elem<T>::pairs(raw, f);
#pragma unroll
    for (int i = 0; i < Elem<T>::kVec / 2; ++i) {
        float2 d = mul2(add2(f[i], minus), scale);
        if (ENT) d = make_float2(max_nan(d.x, -1000.f), max_nan(d.y, -1000.f));
        f[i] = mul2(make_float2(ex2(d.x), ex2(d.y)), ENT ? fma2(k1, d, k0) : k0);
    }
    return Elem<T>::pack(f);
}

// Granules g, g + step, ... of a row below `limit`; `entropy`: k1 is not zero (the same for the whole block).
template <class T, int U>
__device__ __forceinline__ void write_gradient(const uint4 *raw, const Row<T> &row, T *out, bool same, int g, int step, int limit, float c, const RowGrad &k, bool entropy)
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int gu = g + u * step;
        if (gu >= limit) continue;
        row.store(out, same, gu, entropy ? gradient_of<T, true>(raw[u], c, k) : gradient_of<T, false>(raw[u], c, k));
    }
}

// The given token's element: its share of 2^d (k0 + k1 d) plus `hit`, written again by one thread behind a barrier.
template <class T> __device__ __forceinline__ void write_token_gradient(T *out, int token, float x, float c, const RowGrad &k, float hit)
{
    const float d = max_nan((x - k.m) * c, -1000.f);
    out[token] = Elem<T>::from_float(fmaf(ex2(d), fmaf(k.k1, d, k.k0), hit));
}

// The elements of the teacher's set that lie in [e0, e1): A p - (sum of q with this id), written by the thread of the id's
// first entry.  Behind a barrier after the row's other elements were written.
template <class T, int NT>
__device__ __forceinline__ void write_set_gradient(const TeacherShared &sh, int K, T *out, int e0, int e1, float c, float m, float p_scale,
                                                   float q_scale)
{
    for (int j = threadIdx.x; j < K; j += NT) {
        const int32_t id = sh.id[j];
        if (id < 0 || id < e0 || id >= e1) continue;
        float q = 0.f;
        bool first = true;
        for (int i = 0; i < K; ++i) {
            if (sh.id[i] != id) continue;
            if (i < j) first = false;
            q += sh.q[i];
        }
        if (first) out[id] = Elem<T>::from_float(ex2((sh.x[j] - m) * c) * p_scale - q * q_scale);
    }
}

// Gradients from saved sums: one read and one write of the row, a.segments blocks per row.
template <class T, int NT, int U, bool TEACHER, bool TAIL>
__global__ void __launch_bounds__(NT) loss_backward_kernel(const LossArgs a)
{
    __shared__ typename std::conditional<TEACHER, TeacherShared, int>::type shared;
    const int64_t r = blockIdx.x / a.segments;
    const int part = static_cast<int>(blockIdx.x % a.segments);
    const Row<T> row(static_cast<const T *>(a.logits) + r * a.ld, a.V);
    T *out = static_cast<T *>(a.dlogits) + r * a.lddl;
    const int G = row.granules(), per = (G + a.segments - 1) / a.segments;
    const int g0 = min(G, part * per), g1 = min(G, g0 + per);
    const float lse = a.in_lse[r];
    RowGrad k = {0.f, 0.f, 0.f};
    int token = -1;  // V stands for any id beyond the vocabulary
    float hit = 0.f, p_m = 0.f, p_scale = 0.f, q_scale = 0.f;
    if constexpr (TEACHER) {
        teacher_read<T, NT>(shared, a, r, row.first(g0), row.first(g1));
        __syncthreads();
        if (threadIdx.x < 32) teacher_weights<TAIL>(shared, a.K);
        __syncthreads();
        float g = a.grad[r] * a.inv_t;
        if (shared.bad) g = quiet_nan();
        const bool empty = lse == neg_inf();
        p_m = empty ? 0.f : lse * a.temperature;
        if (TAIL) {
            const float rest = a.in_rest[r];
            const bool none = rest == neg_inf();
            const float mass = shared.mass + (none ? 0.f : shared.left);
            k.m = none ? 0.f : rest * a.temperature;
            k.k0 = none ? 0.f : g * fmaf(mass, expf(rest - lse), -shared.left);
            p_scale = g * mass;
        } else {
            k.m = p_m;
            k.k0 = p_scale = g * shared.mass;
        }
        q_scale = g;
        if (empty) k.k0 = p_scale = q_scale = shared.bad ? quiet_nan() : 0.f;
        if (shared.bad) k.k0 = quiet_nan();
    } else {
        const float gh = a.grad_entropy ? a.grad_entropy[r] * a.inv_t : 0.f;
        float gl = 0.f;
        if (a.grad) {
            token = token_at(a, r);
            if (token >= 0) gl = token >= a.V ? quiet_nan() : a.grad[r] * a.inv_t;
            hit = gl;
        }
        if (lse == neg_inf()) {
            k.k0 = hit = token >= a.V ? quiet_nan() : 0.f;
        } else {
            k.m = lse * a.temperature;
            k.k0 = -(a.grad_entropy ? fmaf(gh, a.in_entropy[r], gl) : gl);
            k.k1 = -gh * kLn2;
        }
    }
    const bool same = row.same_lead(out), entropy = k.k1 != 0.f;
    float token_x = 0.f;
    const bool token_here = token >= 0 && token < a.V && token >= row.first(g0) && token < row.first(g1);
    if (!TEACHER && token_here && threadIdx.x == 0) token_x = Elem<T>::to_float(row.p[token]);
    if (!TEACHER) __syncthreads();  // read before it is overwritten in place
    for (int g = g0 + threadIdx.x; g < g1; g += NT * U) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = row.load_below(g + u * NT, g1);
        write_gradient<T, U>(raw, row, out, same, g, NT, g1, a.c, k, entropy);
    }
    __syncthreads();
    if constexpr (TEACHER) {
        write_set_gradient<T, NT>(shared, a.K, out, row.first(g0), row.first(g1), a.c, p_m, p_scale, q_scale);
    } else {
        if (token_here && threadIdx.x == 0) write_token_gradient<T>(out, token, token_x, a.c, k, hit);
    }
}

// Loss and gradient of rows that a cluster holds in registers: U granules per thread, read once.
template <int NT> struct ResidentShared {
    Stats part[NT / 32];
    Stats pub;
    Stats total;
    float loss;
};

template <class T, int NT, int U, bool TEACHER, bool TAIL>
__global__ void __launch_bounds__(NT, 768 / NT) loss_resident_kernel(const LossArgs a)
{
    constexpr bool ENT = !TEACHER;
    __shared__ ResidentShared<NT> sh;
    __shared__ typename std::conditional<TEACHER, TeacherShared, int>::type teacher;
    __shared__ uint32_t bitmap[TAIL ? NT * U * Elem<T>::kVec / 32 : 1];
    cg::cluster_group cluster = cg::this_cluster();
    const int C = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int64_t r = blockIdx.x / C;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Row<T> row(static_cast<const T *>(a.logits) + r * a.ld, a.V);
    T *out = static_cast<T *>(a.dlogits) + r * a.lddl;
    const int G = row.granules(), per = (G + C - 1) / C;
    const int g0 = min(G, rank * per), g1 = min(G, g0 + per);

    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = row.load_below(g0 + u * NT + tid, g1);
    Running run = {neg_inf(), both(0.f), both(0.f)};
    float mi = neg_inf(), si = 0.f;
    int token = -1;
    float token_x = 0.f;
    if constexpr (TEACHER) {
        teacher_read<T, NT>(teacher, a, r, rank == 0 ? 0 : row.first(g0), rank == 0 ? a.V : row.first(g1));
        if (TAIL)
            for (int i = tid; i < NT * U * Elem<T>::kVec / 32; i += NT) bitmap[i] = 0;
        __syncthreads();
        if (warp == 0) teacher_weights<TAIL>(teacher, a.K);
        if (TAIL) {
            for (int j = tid; j < a.K; j += NT) {
                const int pos = teacher.id[j] - row.first(g0);
                if (teacher.id[j] >= 0 && pos >= 0 && pos < (g1 - g0) * Elem<T>::kVec) {
                    const uint32_t bit = 1u << (pos & 31);
                    if (!(atomicOr(&bitmap[pos >> 5], bit) & bit)) add_logit(mi, si, teacher.x[j], a.c);
                }
            }
        }
        __syncthreads();
        if (TAIL) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int g = g0 + u * NT + tid;
                const uint32_t bits = g < g1 ? bits_of<T>(bitmap, g - g0) : 0u;
                if (bits) raw[u] = without<T>(raw[u], bits);
            }
        }
    } else {
        if (a.ids) {
            token = token_at(a, r);
            if (token >= 0 && token < a.V) token_x = Elem<T>::to_float(row.p[token]);
        }
    }
    float all = Elem<T>::max_of(raw[0]);
#pragma unroll
    for (int u = 1; u < U; ++u) all = fmaxf(all, Elem<T>::max_of(raw[u]));
    raise<ENT>(run, all, a.c);
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (g0 + u * NT + (warp << 5) < g1) accumulate<T, ENT>(raw[u], a.c, run);
    Stats st = block_stats<ENT, TAIL, NT>(run, mi, si, sh.part, a.c);
    if (tid == 0) sh.pub = st, sh.total = st;
    if (C > 1) {
        cluster.sync();
        if (warp == 0) {
            st = lane < C ? *cluster.map_shared_rank(&sh.pub, lane) : Stats{neg_inf(), 0.f, 0.f, neg_inf(), 0.f};
#pragma unroll
            for (int d = 4; d; d >>= 1) join_stats<ENT, TAIL>(st, shuffle_xor<ENT, TAIL>(st, d), a.c);
            if (lane == 0) sh.total = st;
        }
        cluster.sync();  // the peers have read; from here on every block is on its own
    } else {
        __syncthreads();
    }
    st = sh.total;
    const RowEnd e = row_end<TAIL>(st, a.c);
    RowGrad k = {0.f, 0.f, 0.f};
    float hit = 0.f, p_m = 0.f, p_scale = 0.f, q_scale = 0.f;
    if constexpr (TEACHER) {
        if (rank == 0 && warp == 0) {
            const float loss = teacher_loss<TAIL>(teacher, e, a.inv_t, a.K);
            if (lane == 0) {
                if (a.loss) a.loss[r] = loss;
                if (a.lse) a.lse[r] = lse_of(e.m, e.ls, e.empty, a.inv_t);
                if (TAIL && a.rest) a.rest[r] = lse_of(e.mr, e.lsr, e.rest_empty, a.inv_t);
            }
        }
        const float g = teacher.bad ? quiet_nan() : a.grad[r] * a.inv_t;
        const float inv_s = 1.f / e.s;
        p_m = e.empty ? 0.f : e.m;
        const float mass = teacher.mass + (TAIL && !e.rest_empty ? teacher.left : 0.f);
        p_scale = g * mass * inv_s;
        if (TAIL) {
            k.m = e.rest_empty ? 0.f : e.mr;
            k.k0 = e.rest_empty ? 0.f : g * fmaf(mass, ex2((e.mr - e.m) * a.c) * e.sr * inv_s, -teacher.left) / e.sr;
        } else {
            k.m = p_m, k.k0 = p_scale;
        }
        q_scale = g;
        if (e.empty) k.k0 = p_scale = q_scale = 0.f;
        if (teacher.bad) k.k0 = p_scale = q_scale = quiet_nan();
    } else {
        const float mean_d = e.empty ? 0.f : st.t / st.s;  // sum p d
        if (rank == 0 && tid == 0) {
            if (a.lse) a.lse[r] = lse_of(e.m, e.ls, e.empty, a.inv_t);
            if (a.entropy) a.entropy[r] = e.empty ? 0.f : kLn2 * (e.ls - mean_d);
            if (a.logprob) {
                float lp = 0.f;
                if (token >= a.V) lp = quiet_nan();
                else if (token >= 0) lp = log_prob(token_x, e, a.inv_t);
                a.logprob[r] = lp;
            }
        }
        const float gh = a.grad_entropy ? a.grad_entropy[r] * a.inv_t : 0.f;
        float gl = 0.f;
        if (a.grad && token >= 0) gl = token >= a.V ? quiet_nan() : a.grad[r] * a.inv_t;
        hit = gl;
        if (e.empty) {
            k.k0 = hit = a.grad && token >= a.V ? quiet_nan() : 0.f;
        } else {
            // p (gl + gh (log p + H)) with log p + H = ln 2 (d - mean_d)
            const float inv_s = 1.f / st.s;
            k.m = e.m;
            k.k0 = -fmaf(-gh * kLn2, mean_d, gl) * inv_s;
            k.k1 = -gh * kLn2 * inv_s;
        }
    }
    // the elements are unpacked again rather than kept unpacked in twice the registers
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" : "+r"(raw[u].x), "+r"(raw[u].y), "+r"(raw[u].z), "+r"(raw[u].w));
    write_gradient<T, U>(raw, row, out, row.same_lead(out), g0 + tid, NT, g1, a.c, k, k.k1 != 0.f);
    __syncthreads();
    if constexpr (TEACHER) {
        write_set_gradient<T, NT>(teacher, a.K, out, row.first(g0), row.first(g1), a.c, p_m, p_scale, q_scale);
    } else {
        if (tid == 0 && token >= 0 && token < a.V && token >= row.first(g0) && token < row.first(g1)) write_token_gradient<T>(out, token, token_x, a.c, k, hit);
    }
}

// ------------------------------------------------------------------------------------------ launches
template <class T> inline int64_t most_granules(int64_t V) { return (V + Elem<T>::kVec - 1) / Elem<T>::kVec + 1; }

template <class Kernel> inline int launch_clusters(Kernel kernel, int64_t rows, int cluster, int threads, size_t smem, cudaStream_t stream, const LossArgs &a)
{
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>(rows * cluster));
    config.blockDim = dim3(static_cast<unsigned>(threads));
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = cluster > 1 ? 1 : 0;
    SPDY_EVAL_TRY(cudaLaunchKernelEx(&config, kernel, a));
    return SPDY_OK;
}

constexpr int64_t kMostBlocks = 0x7fffffff;

template <class T, int NT, int MODE> inline int forward_with(const LossArgs &a, int cluster, cudaStream_t stream)
{
    size_t smem = 0;
    if (MODE == kDistill) smem = sizeof(TeacherShared);
    if (MODE == kDistillTail) smem = sizeof(TeacherShared) + 4 * kBitmapWords;
    if (MODE == kLogprobsTop) {
        const int64_t steps = (most_granules<T>(a.V) / cluster + NT * 4) / (NT * 4);
        smem = sizeof(TopShared) + sizeof(uint32_t) * NT * static_cast<size_t>(steps < kGroupSteps ? steps + 1 : kGroupSteps + 1);
        SPDY_EVAL_TRY(cudaFuncSetAttribute(loss_forward_kernel<T, NT, 4, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           static_cast<int>(sizeof(TopShared) + sizeof(uint32_t) * NT * (kGroupSteps + 1))));
    }
    return launch_clusters(loss_forward_kernel<T, NT, 4, MODE>, a.R, cluster, NT, smem, stream, a);
}

template <class T, int MODE> int forward(const LossArgs &a, cudaStream_t stream)
{
    // Short rows get small blocks, so that many rows are in flight on a multiprocessor; a row is divided among up to eight
    // blocks when the rows alone would not fill the device twice and every block still has a step of work.
    const int64_t G = most_granules<T>(a.V);
    const bool small = G <= 512;
    int cluster = 1;
    while (cluster < 8 && a.R * cluster < 2 * sm_count() && G > static_cast<int64_t>(cluster) * (small ? 512 : 1024)) cluster *= 2;
    if (a.R * cluster > kMostBlocks) return SPDY_ERR_UNSUPPORTED;
    return small ? forward_with<T, 128, MODE>(a, cluster, stream) : forward_with<T, 256, MODE>(a, cluster, stream);
}

template <class T, bool TEACHER, bool TAIL> int backward(LossArgs a, cudaStream_t stream)
{
    constexpr int NT = 256, U = 4;
    const int64_t G = most_granules<T>(a.V);
    a.segments = static_cast<int>((G + 2 * NT * U - 1) / (2 * NT * U));
    if (a.R * a.segments < 4 * sm_count()) a.segments = static_cast<int>((G + NT - 1) / NT);
    if (a.R * a.segments > kMostBlocks) return SPDY_ERR_UNSUPPORTED;
    loss_backward_kernel<T, NT, U, TEACHER, TAIL><<<static_cast<unsigned>(a.R * a.segments), NT, 0, stream>>>(a);
    return finish_launch();
}

// Whether a cluster holds the row in registers; if so, loss and gradient in one launch.
template <class T, bool TEACHER, bool TAIL> int resident(const LossArgs &a, cudaStream_t stream, bool &fits)
{
    constexpr int U = 8;
    const int64_t G = most_granules<T>(a.V);
    fits = G <= 8 * 512 * U;
    if (!fits) return SPDY_OK;
    const int NT = G <= 128 * U ? 128 : G <= 8 * 256 * U ? 256 : 512;
    int cluster = static_cast<int>((G + NT * U - 1) / (NT * U));
    while (cluster < 8 && a.R * cluster < sm_count() && G > static_cast<int64_t>(cluster) * NT) ++cluster;
    if (a.R * cluster > kMostBlocks) return SPDY_ERR_UNSUPPORTED;
    if (NT == 128) return launch_clusters(loss_resident_kernel<T, 128, U, TEACHER, TAIL>, a.R, cluster, NT, 0, stream, a);
    if (NT == 256) return launch_clusters(loss_resident_kernel<T, 256, U, TEACHER, TAIL>, a.R, cluster, NT, 0, stream, a);
    return launch_clusters(loss_resident_kernel<T, 512, U, TEACHER, TAIL>, a.R, cluster, NT, 0, stream, a);
}

#define SPDY_EVAL_BY_TYPE(dtype, call)                                                          \
    ((dtype) == SPDY_F32 ? [&] { using T = float; return call; }()                              \
     : (dtype) == SPDY_BF16 ? [&] { using T = __nv_bfloat16; return call; }()                   \
                            : [&] { using T = __half; return call; }())

constexpr int64_t kMostColumns = 0x7fffffff - 64;

inline bool rows_ok(const void *p, int64_t ld, int dtype, int64_t R, int64_t V)
{
    return known_type(dtype) && R >= 0 && V >= 1 && V <= kMostColumns && ld >= V && (R == 0 || (p && aligned(p, type_size(dtype))));
}
inline bool temperature_ok(float t) { return t > 0.f && t <= 3.4e38f && kLog2e / t <= 3.4e38f && kLog2e / t > 0.f; }

}  // namespace spdy_eval
#endif
