// Kernels over rows of logits: log probabilities of given tokens (with entropy and top alternatives), the distillation
// loss, and their gradients.  Instantiated in eval_token_logprobs.cu and eval_distill.cu.
//
// Mathematics.  Everything is kept in base 2: with c = log2(e) / T and the running maximum m of the logits, d_v = (x_v - m) c
// and s = sum 2^d, a probability is 2^d_v / s.  The entropy needs t = sum 2^d d beside s: H = ln 2 (log2 s - t / s).  When the
// maximum rises by delta / c, s becomes s 2^-delta and t becomes (t - s delta) 2^-delta.
// m need not be the maximum: any logit within a factor of 4 of it does (see raise), so that the sums are rescaled
// rarely and nothing large cancels in the end.
// An element costs one fused multiply-add x c - b with b = m c rounded; the rounding r = m c - b is the same for all elements and
// is taken back once per thread (2^-r s, and t - r s for t).  From |m c| = 2^24 on, where r could reach 1 and soon what 2^r
// overflows at (masks of -1e9, tiny temperatures), m is subtracted first instead.  Beside that one instruction to unpack, one for the special-function unit
// (16 results a cycle and multiprocessor) and one or two to add up.
//
// Bound.  Rows are read once, and with a gradient written once.  At 4 to 6 bytes moved and 8 to 20 instructions issued per element the
// issue slots (65 to 75 % taken) and memory (50 to 65 %) are loaded alike; rows of a few thousand elements add their ends: some hundred
// instructions per thread to join the sums and the teacher's entries.
// Measured, bf16, us (and the bytes at 6.56 TB/s): 2048 x 131072 log probabilities 94 (82), with the best 20 128, with
// gradient 220 (164), distillation from 32 ids 94, with gradient 220; 4096 x 65536 104 (82), 124, 214 (164), 106, 215; 1024 x 50001 (rows
// that start anywhere) 28 (16), 36, 55 (31), 31, 57; 16384 x 8192 72 (41), 139, 109 (82), 89, 144; 65536 x 2000 62 (40), 176, 115 (80),
// 113, 192.  Backward passes from saved sums: 159, 159, 37, 84, 98 and 200, 204, 50, 102, 144.  Masks of -inf cost nothing: 95 % of
// 8192 x 30000 118, of 65536 x 2000 62.
#ifndef SPDY_EVAL_LOSS_CUH
#define SPDY_EVAL_LOSS_CUH

#include <algorithm>
#include <type_traits>

#include "eval_common.cuh"
#include "eval_top.cuh"

namespace spdy_eval {

namespace cg = cooperative_groups;

struct LossArgs {
    const void *logits;
    int64_t ld, R, V;
    float c, inv_t, temperature;  // c = log2(e) / T
    float lower;             // saved_reference
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
    int per_block, steps;    // granules of a row that one of a cluster's blocks takes, and their steps (of the longest row)
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

// What 2^(x c - base) is relative to: base = m c rounded (off by at most 1/2), or, far from 0, m c itself after subtracting
// sub = m.  With m = -inf there is nothing yet: base is 0, and ids that are not allowed give 2^-inf.
constexpr float kFar = 16777216.f;
struct Reference {
    float base, sub;
    bool far;
    __device__ __forceinline__ Reference(float m, float c)
    {
        base = m == neg_inf() ? 0.f : m * c;
        far = !(fabsf(base) < kFar);  // also m = +inf and NaN
        sub = far ? m : 0.f;
        if (far) base = 0.f;
    }
};

// What a thread has added up, relative to Reference(m, c): m is some logit, no other is more than 2 / c above it.
struct Running {
    float m, s, t;
};

// Makes `top` the logit the sums are relative to, if it is far above the present one (or the first).
template <bool ENT> __device__ __forceinline__ void raise(Running &st, float top, float c)
{
    if ((top - st.m) * c > 2.f) {  // not so where both are -inf, or one is NaN
        if (st.s != 0.f) {
            const Reference old(st.m, c), now(top, c);
            const float rise = old.far ? (now.far ? (st.m - top) * c : fmaf(st.m, c, -now.base)) : now.far ? -fmaf(top, c, -old.base) : old.base - now.base;
            const float d = max_nan(rise, -1000.f), f = ex2(d);
            if (ENT) st.t = f * fmaf(st.s, d, st.t);
            st.s *= f;
        }
        st.m = top;
    }
}

// Adds a granule's elements with any reference: out of line, it is rare.
template <class T> __device__ __noinline__ Running accumulate_far(uint4 raw, float c, Running st)
{
    const Reference ref(st.m, c);
    float f[Elem<T>::kVec];
    Elem<T>::unpack(raw, f);
#pragma unroll
    for (int i = 0; i < Elem<T>::kVec; ++i) {
        const float d = max_nan(ref.far ? (f[i] - ref.sub) * c : fmaf(f[i], c, -ref.base), -1000.f), e = ex2(d);
        st.s += e;
        st.t = fmaf(e, d, st.t);
    }
    return st;
}

// Adds U granules of each thread of a warp, after raise.
template <class T, int U, bool ENT> __device__ __forceinline__ void accumulate(const uint4 *raw, float c, Running &st)
{
    const Reference ref(st.m, c);
    if (__any_sync(0xffffffffu, ref.far)) {
#pragma unroll
        for (int u = 0; u < U; ++u) st = accumulate_far<T>(raw[u], c, st);
        return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[Elem<T>::kVec];
        Elem<T>::unpack(raw[u], f);
#pragma unroll
        for (int i = 0; i < Elem<T>::kVec; ++i) {
            float d = fmaf(f[i], c, -ref.base);
            if (ENT) d = max_nan(d, -1000.f);  // an id that is not allowed adds 0 rather than 0 times -inf
            const float e = ex2(d);
            st.s += e;
            if (ENT) st.t = fmaf(e, d, st.t);
        }
    }
}

// The sums relative to m itself.
template <bool ENT> __device__ __forceinline__ void settle(Running &st, float c)
{
    const Reference ref(st.m, c);
    if (ref.far || st.s == 0.f) return;
    const float r = fmaf(st.m, c, -ref.base), f = ex2(-r);
    if (ENT) st.t = f * fmaf(-r, st.s, st.t);
    st.s *= f;
}

// -inf in place of the elements whose bit is set
template <class T> __device__ __forceinline__ uint4 without(uint4 raw, uint32_t bits)
{
    constexpr uint32_t NI = Elem<T>::kNegInfWord;
    if (sizeof(T) == 4) return make_uint4(bits & 1 ? NI : raw.x, bits & 2 ? NI : raw.y, bits & 4 ? NI : raw.z, bits & 8 ? NI : raw.w);
    const auto word = [](uint32_t w, uint32_t two) {
        const uint32_t mask = (two & 1 ? 0xffffu : 0u) | (two & 2 ? 0xffff0000u : 0u);
        return (w & ~mask) | (NI & mask);
    };
    return make_uint4(word(raw.x, bits), word(raw.y, bits >> 2), word(raw.z, bits >> 4), word(raw.w, bits >> 6));
}

// The bits of granule g (counted from the first one the bitmap covers).
template <class T> __device__ __forceinline__ uint32_t bits_of(const uint32_t *bitmap, int g)
{
    if (Elem<T>::kVec == 8) return reinterpret_cast<const uint8_t *>(bitmap)[g];
    return reinterpret_cast<const uint8_t *>(bitmap)[g >> 1] >> ((g & 1) * 4) & 15u;
}

// ------------------------------------------------------------------------------------------ teacher's entries
struct TeacherShared {
    int32_t id[SPDY_DISTILL_MAX];  // -1: no entry
    float q[SPDY_DISTILL_MAX], logq[SPDY_DISTILL_MAX];
    float x[SPDY_DISTILL_MAX];     // the student's logit at id
    float left, mass;              // mass: sum of q
    int bad;                       // an id >= V
    int twice;                     // an id may come twice
};

// What a thread of n holds of a row's entries: those t, t + n, ...  Ids and log probabilities are on their way from the
// constructor on; the student's logits follow from `place` and are put down by `settle`, so that a row need not wait for them
// before it is streamed.
template <class T, int N> struct Entries {
    static constexpr int kEach = (SPDY_DISTILL_MAX + N - 1) / N;
    int64_t id[kEach];
    float logq[kEach], x[kEach];

    __device__ __forceinline__ Entries(const LossArgs &a, int64_t row, int t)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = i * N + t;
            id[i] = j < a.K ? index_at(a.ids, a.index_bits, row * a.K + j) : -1;
            logq[i] = j < a.K ? a.top_lp[row * a.K + j] : 0.f;
        }
    }
    // The student's logits only for ids in [e0, e1) (another block may be overwriting the rest in place).
    __device__ __forceinline__ void place(TeacherShared &sh, const LossArgs &a, int64_t row, int e0, int e1, int t)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = i * N + t;
            if (j >= a.K) break;
            const bool here = id[i] >= 0 && id[i] < a.V;
            if (id[i] >= a.V) sh.bad = 1;
            sh.id[j] = here ? static_cast<int32_t>(id[i]) : -1;
            sh.logq[j] = here ? logq[i] : neg_inf();
            x[i] = here && id[i] >= e0 && id[i] < e1 ? Elem<T>::to_float(static_cast<const T *>(a.logits)[row * a.ld + id[i]]) : neg_inf();
        }
    }
    // place without the student's logits, which `gather` fetches later (they cost registers meanwhile).
    __device__ __forceinline__ void place_ids(TeacherShared &sh, const LossArgs &a, int t) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = i * N + t;
            if (j >= a.K) break;
            const bool here = id[i] >= 0 && id[i] < a.V;
            if (id[i] >= a.V) sh.bad = 1;
            sh.id[j] = here ? static_cast<int32_t>(id[i]) : -1;
            sh.logq[j] = here ? logq[i] : neg_inf();
        }
    }
    __device__ __forceinline__ void gather(const TeacherShared &sh, int K, const T *row, int e0, int e1, int t)
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = i * N + t;
            if (j >= K) break;
            const int at = sh.id[j];
            x[i] = at >= 0 && at >= e0 && at < e1 ? Elem<T>::to_float(row[at]) : neg_inf();
        }
    }
    __device__ __forceinline__ void settle(TeacherShared &sh, int K, int t) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (i * N + t < K) sh.x[i * N + t] = x[i];
    }
    // Marks the ids among elements first .. first + count - 1 in a bitmap; bit i of the result: entry i was the first to mark its id.
    __device__ __forceinline__ uint32_t mark(TeacherShared &sh, int K, uint32_t *bitmap, int first, int count, int t) const
    {
        uint32_t marked = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = i * N + t;
            if (j >= K) break;
            const int pos = sh.id[j] - first;
            if (sh.id[j] < 0 || pos < 0 || pos >= count) continue;
            const uint32_t bit = 1u << (pos & 31);
            if (atomicOr(&bitmap[pos >> 5], bit) & bit) sh.twice = 1;
            else marked |= 1u << i;
        }
        return marked;
    }
    __device__ __forceinline__ void unmark(const TeacherShared &sh, int K, uint32_t *bitmap, int first, int count, int t) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = i * N + t;
            if (j >= K) break;
            const int pos = sh.id[j] - first;
            if (sh.id[j] >= 0 && pos >= 0 && pos < count) bitmap[pos >> 5] = 0;
        }
    }
    // Adds the logits of the entries that marked their ids to the sums over the set.
    __device__ __forceinline__ void add_marked(uint32_t marked, float c, float &mi, float &si) const
    {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (marked >> i & 1) add_logit(mi, si, x[i], c);
    }
};

// q, log q, left and mass from the entries; one warp, after a barrier behind Entries::place.
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

// ------------------------------------------------------------------------------------------ results and gradients of a row
enum { kLogprobs = 0, kLogprobsTop = 1, kDistill = 2, kDistillTail = 3 };
enum { kNoGrad = 0, kGrad = 1, kGradSaved = 2 };  // no gradient; from this call's sums; from a forward call's

template <bool ENT, bool TAIL> __device__ __forceinline__ Stats warp_stats(Running run, float mi, float si, float c)
{
    settle<ENT>(run, c);
    // the warp's largest reference first, so that every lane rescales once and the rest are additions
    Stats st = {warp_max(run.m), run.s, run.t, mi, si};
    if (st.s != 0.f) {
        const float d = max_nan((run.m - st.m) * c, -1000.f), f = ex2(d);
        if (ENT) st.t = f * fmaf(st.s, d, st.t);
        st.s *= f;
    }
    st.s = warp_sum(st.s);
    if (ENT) st.t = warp_sum(st.t);
    if (TAIL) {
        st.mi = warp_max(mi);
        if (si != 0.f) st.si = si * ex2((mi - st.mi) * c);
        st.si = warp_sum(st.si);
    }
    return st;
}

struct NoEntries {
    __device__ __forceinline__ NoEntries(const LossArgs &, int64_t, int) {}
};

// One thread writes a row's sums; `token_x` is the given token's logit.
template <bool ENT, bool TAIL> __device__ __forceinline__ void write_sums(const LossArgs &a, int64_t r, const Stats &st, const RowEnd &e, int token, float token_x)
{
    if (a.lse) a.lse[r] = lse_of(e.m, e.ls, e.empty, a.inv_t);
    if (ENT) {
        if (a.entropy) a.entropy[r] = e.empty ? 0.f : kLn2 * (e.ls - st.t / st.s);
        if (a.logprob) a.logprob[r] = token < 0 ? 0.f : token >= a.V ? quiet_nan() : log_prob(token_x, e, a.inv_t);
    }
    if (TAIL && a.rest) a.rest[r] = lse_of(e.mr, e.lsr, e.rest_empty, a.inv_t);
}

// A row's gradient: 2^d (k0 + k1 d) with d = (x - m) c for every element, `hit` more for the given token, and for the
// teacher's ids 2^((x - p_m) c) p_scale - q q_scale instead.
struct RowGrad {
    float m, k0, k1, hit;
    float p_m, p_scale, q_scale;
};

template <bool TAIL> __device__ __forceinline__ RowGrad teacher_gradient(const LossArgs &a, int64_t r, const RowEnd &e, const TeacherShared &teacher)
{
    RowGrad k = {};
    const float g = teacher.bad ? quiet_nan() : a.grad[r] * a.inv_t;
    const float inv_s = 1.f / e.s;
    const float mass = teacher.mass + (TAIL && !e.rest_empty ? teacher.left : 0.f);
    k.p_m = e.empty ? 0.f : e.m;
    k.p_scale = g * mass * inv_s;
    k.q_scale = g;
    if (TAIL) {
        k.m = e.rest_empty ? 0.f : e.mr;
        k.k0 = e.rest_empty ? 0.f : g * fmaf(mass, ex2((e.mr - e.m) * a.c) * e.sr * inv_s, -teacher.left) / e.sr;
    } else {
        k.m = k.p_m, k.k0 = k.p_scale;
    }
    if (e.empty) k.k0 = k.p_scale = k.q_scale = 0.f;
    if (teacher.bad) k.k0 = k.p_scale = k.q_scale = quiet_nan();
    return k;
}

// The logit that a saved lse stands for.  Far from 0 the last place of lse may be worth more than the row's whole sum: there it is
// lowered by the roundings on the way (the quotient's, the sum's, the product's), so that the row's largest logits are not below
// it, and p is counted at most 1 (exponent).
__device__ __forceinline__ float saved_reference(const LossArgs &a, float lse)
{
    const float m = lse * a.temperature;
    return max_nan(fmaf(-fabsf(m), fabsf(m * a.c) < kFar ? 0.f : a.lower, m), -3.4028235e38f);
}
template <bool SAVED> __device__ __forceinline__ float exponent(float x, float m, float c)
{
    return SAVED ? min_nan((x - m) * c, 0.f) : (x - m) * c;
}

template <bool TAIL> __device__ __forceinline__ RowGrad teacher_gradient_saved(const LossArgs &a, int64_t r, const TeacherShared &teacher)
{
    RowGrad k = {};
    const float lse = a.in_lse[r], g = teacher.bad ? quiet_nan() : a.grad[r] * a.inv_t;
    const bool empty = lse == neg_inf();
    k.p_m = empty ? 0.f : saved_reference(a, lse);
    if (TAIL) {
        const float rest = a.in_rest[r];
        const bool none = rest == neg_inf();
        const float mass = teacher.mass + (none ? 0.f : teacher.left);
        k.m = none ? 0.f : saved_reference(a, rest);
        const float over = rest - lse;  // above 0 by its roundings alone
        k.k0 = none ? 0.f : g * fmaf(mass, over > 0.f ? 1.f : expf(over), -teacher.left);
        k.p_scale = g * mass;
    } else {
        k.m = k.p_m;
        k.k0 = k.p_scale = g * teacher.mass;
    }
    k.q_scale = g;
    if (empty) k.k0 = k.p_scale = k.q_scale = 0.f;
    if (teacher.bad) k.k0 = k.p_scale = k.q_scale = quiet_nan();
    return k;
}

__device__ __forceinline__ float token_weight(const LossArgs &a, int64_t r, int token)
{
    if (!a.grad || token < 0) return 0.f;
    return token >= a.V ? quiet_nan() : a.grad[r] * a.inv_t;
}

// p (gl + gh (log p + H)) with log p + H = ln 2 (d - sum p d)
__device__ __forceinline__ RowGrad token_gradient(const LossArgs &a, int64_t r, const Stats &st, const RowEnd &e, int token)
{
    RowGrad k = {};
    const float gh = a.grad_entropy ? a.grad_entropy[r] * a.inv_t : 0.f, gl = token_weight(a, r, token);
    k.hit = gl;
    if (e.empty) {
        k.k0 = k.hit = gl != gl ? gl : 0.f;
    } else {
        const float inv_s = 1.f / st.s;
        k.m = e.m;
        k.k0 = -fmaf(-gh * kLn2, st.t * inv_s, gl) * inv_s;
        k.k1 = -gh * kLn2 * inv_s;
    }
    return k;
}

__device__ __forceinline__ RowGrad token_gradient_saved(const LossArgs &a, int64_t r, int token)
{
    RowGrad k = {};
    const float lse = a.in_lse[r], gh = a.grad_entropy ? a.grad_entropy[r] * a.inv_t : 0.f, gl = token_weight(a, r, token);
    k.hit = gl;
    if (lse == neg_inf()) {
        k.k0 = k.hit = gl != gl ? gl : 0.f;
    } else {
        k.m = saved_reference(a, lse);
        k.k0 = -(a.grad_entropy ? fmaf(gh, a.in_entropy[r], gl) : gl);
        k.k1 = -gh * kLn2;
    }
    return k;
}

// A row's factors relative to Reference(m, c) (compare settle).
struct Factors {
    Reference ref;
    float k0, k1;
    __device__ __forceinline__ Factors(const RowGrad &k, float c) : ref(k.m, c)
    {
        const float r = ref.far ? 0.f : fmaf(k.m, c, -ref.base), f = ex2(-r);
        k0 = f * fmaf(-r, k.k1, k.k0);
        k1 = f * k.k1;
    }
};

// How a row's elements are turned into their gradients and written.
template <class T, bool ENT, bool SAVED> struct GradientWriter {
    T *out;
    bool same, entropy;
    float base, k0, k1;
    const Factors &all;  // for the rare rest
    __device__ __forceinline__ GradientWriter(const Row<T> &row, T *to, const Factors &f)
        : out(to), same(row.same_lead(to)), entropy(ENT && f.k1 != 0.f), base(f.ref.base), k0(f.k0), k1(f.k1), all(f)
    {
    }
    template <bool ENTROPY> __device__ __forceinline__ uint4 gradient(uint4 raw, float c) const
    {
        float f[Elem<T>::kVec];
        Elem<T>::unpack(raw, f);
#pragma unroll
        for (int i = 0; i < Elem<T>::kVec; ++i) {
            float d = fmaf(f[i], c, -base);
            if (ENTROPY) {
                d = max_nan(d, -1000.f);
                f[i] = ex2(d) * fmaf(k1, d, k0);
            } else {
                f[i] = ex2(d) * k0;
            }
        }
        return Elem<T>::pack(f);
    }
    // A granule's elements one by one, with a far reference.
    static __device__ __noinline__ uint4 far_gradient(uint4 raw, float c, float sub, float k0, float k1)
    {
        float f[Elem<T>::kVec];
        Elem<T>::unpack(raw, f);
#pragma unroll
        for (int i = 0; i < Elem<T>::kVec; ++i) {
            const float d = max_nan(exponent<SAVED>(f[i], sub, c), -1000.f);
            f[i] = ex2(d) * fmaf(k1, d, k0);
        }
        return Elem<T>::pack(f);
    }
    template <int NT, int U> __device__ __forceinline__ void write(const Step<T, NT, U> &step, const uint4 *raw, float c) const
    {
        if (!step.plain || !same || all.ref.far) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (step.g + u * NT < step.limit)
                    step.store_part_of(out, same, u, all.ref.far ? far_gradient(raw[u], c, all.ref.sub, k0, k1) : ENT && entropy ? gradient<true>(raw[u], c) : gradient<false>(raw[u], c));
            return;
        }
        T *to = out + step.row.first(step.g);
        if (ENT && entropy) {
#pragma unroll
            for (int u = 0; u < U; ++u) store_last(to + u * NT * Elem<T>::kVec, gradient<true>(raw[u], c));
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) store_last(to + u * NT * Elem<T>::kVec, gradient<false>(raw[u], c));
        }
    }
};

// The given token's element, written again by one thread behind a barrier.
template <class T, bool SAVED> __device__ __forceinline__ void write_token_gradient(T *out, int token, float x, float c, const RowGrad &k)
{
    const float d = max_nan(exponent<SAVED>(x, k.m, c), -1000.f);
    out[token] = Elem<T>::from_float(fmaf(ex2(d), fmaf(k.k1, d, k.k0), k.hit));
}

// The teacher's ids that lie in [e0, e1), written again behind a barrier by the thread of the id's first entry, by `n` threads.
template <class T, bool SAVED> __device__ __forceinline__ void write_set_gradient(const TeacherShared &sh, int K, T *out, int e0, int e1, float c, const RowGrad &k, int t, int n)
{
    for (int j = t; j < K; j += n) {
        const int32_t id = sh.id[j];
        if (id < 0 || id < e0 || id >= e1) continue;
        float q = sh.q[j];
        bool first = true;
        if (sh.twice) {
            q = 0.f;
#pragma unroll 4
            for (int i = 0; i < K; ++i)
                if (sh.id[i] == id) {
                    first = first && i >= j;
                    q += sh.q[i];
                }
        }
        if (first) out[id] = Elem<T>::from_float(ex2(exponent<SAVED>(sh.x[j], k.p_m, c)) * k.p_scale - q * k.q_scale);
    }
}

// Entries that block `b` of a row's cluster contributes to its alternatives.
template <class T> __device__ __forceinline__ int share_count(const Row<T> &row, int per, int b, int K)
{
    const int G = row.granules(), g0 = min(G, b * per), g1 = min(G, g0 + per);
    return max(0, min(K, min(row.n, row.first(g1)) - max(0, row.first(g0))));
}

// ------------------------------------------------------------------------------------------ short rows: one warp each
constexpr int kWarpRows = 4;         // rows, and warps, of a block
constexpr int kWarpCandidates = 256;

constexpr int kWarpListed = 160;     // granules: the best 128 and some equal ones

struct WarpTop {
    uint4 granule[kWarpListed];
    uint64_t cand[kWarpCandidates + 1];  // the last takes what is too many
    uint16_t index[kWarpListed];
};

template <class T, int U, int MODE> struct WarpShared {
    TeacherShared teacher[MODE >= kDistill ? kWarpRows : 1];
    uint32_t bitmap[MODE >= kDistill ? kWarpRows : 1][U * Elem<T>::kVec];
    WarpTop top[MODE == kLogprobsTop ? kWarpRows : 1];
};

// The `want` best of a warp's granules, as keys in sh.cand[0..n), n <= kWarpCandidates; returns n.  The want-th largest granule's
// largest element (or lane's) bounds the want-th largest element from below.
template <class T, int U> __device__ __forceinline__ int warp_top(uint4 *raw, const Row<T> &row, int G, int want, WarpTop &sh)
{
    uint64_t *const cand = sh.cand;
    constexpr int VEC = Elem<T>::kVec;
    const int lane = threadIdx.x & 31;
    uint32_t keys[U];
#pragma unroll
    for (int u = 0; u < U; ++u) keys[u] = u * 32 + lane < G ? ordered(Elem<T>::max_of(raw[u])) : 0u;
    uint32_t v = 0;
    if (want <= 32) {  // the want-th largest of the lanes' largest will do, a little lower
        uint32_t mine = keys[0];
#pragma unroll
        for (int u = 1; u < U; ++u) mine = max(mine, keys[u]);
        int rank = 0;
#pragma unroll 8
        for (int l = 0; l < 32; ++l) {
            const uint32_t other = __shfl_sync(0xffffffffu, mine, l);
            rank += other > mine || (other == mine && l < lane);
        }
        v = __reduce_max_sync(0xffffffffu, rank == want - 1 ? mine : 0u);
    } else {
        for (int b = 31; b >= (VEC == 8 ? 12 : 0); --b) {  // 16-bit types: the low bits of the order are all alike
            const uint32_t trial = v | 1u << b;
            int n = 0;
#pragma unroll
            for (int u = 0; u < U; ++u) n += keys[u] >= trial;
            if (static_cast<int>(__reduce_add_sync(0xffffffffu, n)) >= want) v = trial;
        }
    }
    // the granules that can hold one of the best are put side by side, so that the lanes share their elements
    const uint32_t below = (1u << lane) - 1u;
    int listed = 0, n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const bool takes = u * 32 + lane < G && (v == 0 || keys[u] >= v);
        const uint32_t mask = __ballot_sync(0xffffffffu, takes);
        const int at = listed + __popc(mask & below);
        if (takes && at < kWarpListed) sh.granule[at] = raw[u], sh.index[at] = static_cast<uint16_t>(u * 32 + lane);
        listed += __popc(mask);
    }
    __syncwarp();
    if (listed <= kWarpListed) {
        for (int i = lane; i - lane < listed * VEC; i += 32) {
            bool takes = false;
            uint64_t key = 0;
            if (i < listed * VEC) {
                const float f = Elem<T>::to_float(reinterpret_cast<const T *>(sh.granule)[i]);
                const int e = row.first(sh.index[i / VEC]) + i % VEC;
                takes = ordered(f) >= v && e >= 0 && e < row.n;
                key = rank_key(f, static_cast<uint32_t>(e));
            }
            const uint32_t mask = __ballot_sync(0xffffffffu, takes);
            if (takes) cand[min(n + __popc(mask & below), kWarpCandidates)] = key;
            n += __popc(mask);
        }
        __syncwarp();
    }
    if (n <= kWarpCandidates && n >= want) return n;
    // many equal or many in few granules (or a bound from beyond the row's end, beside NaN alone): the want-th largest element itself, bit by bit, then those above it and the first
    // ones equal to it
    v = 0;
#pragma unroll 1
    for (int b = 31; b >= 0; --b) {
        const uint32_t trial = v | 1u << b;
        int c = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            asm volatile("" : "+r"(raw[u].x), "+r"(raw[u].y), "+r"(raw[u].z), "+r"(raw[u].w));  // unpacked anew in every round
            const int e = row.first(u * 32 + lane);
            float f[VEC];
            Elem<T>::unpack(raw[u], f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) c += ordered(f[i]) >= trial && e + i >= 0 && e + i < row.n;
        }
        if (static_cast<int>(__reduce_add_sync(0xffffffffu, c)) >= want) v = trial;
    }
    int have = 0;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            asm volatile("" : "+r"(raw[u].x), "+r"(raw[u].y), "+r"(raw[u].z), "+r"(raw[u].w));
            const int e = row.first(u * 32 + lane);
            float f[VEC];
            Elem<T>::unpack(raw[u], f);
            uint32_t bits = 0;
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if ((pass == 0 ? ordered(f[i]) > v : ordered(f[i]) == v) && e + i >= 0 && e + i < row.n) bits |= 1u << i;
            int at = __popc(bits);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int other = __shfl_up_sync(0xffffffffu, at, d);
                if (lane >= d) at += other;
            }
            const int total = __shfl_sync(0xffffffffu, at, 31);
            at += have - __popc(bits);
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (bits >> i & 1) {
                    if (at < want) cand[at] = rank_key(f[i], static_cast<uint32_t>(e + i));
                    ++at;
                }
            have += total;
        }
    }
    __syncwarp();
    return want;
}

// Rows of up to 32 U granules: a warp reads its row once, keeps it in registers and needs no barrier (65536 x 2000 bf16: 64 us; with
// a block of 128 per row 217).
template <class T, int U, int MODE, int GRAD> __global__ void __launch_bounds__(32 * kWarpRows) loss_warp_kernel(const LossArgs a)
{
    constexpr bool ENT = MODE == kLogprobs || MODE == kLogprobsTop, TEACHER = MODE >= kDistill, TAIL = MODE == kDistillTail;
    __shared__ WarpShared<T, U, MODE> sh;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t r = static_cast<int64_t>(blockIdx.x) * kWarpRows + warp;
    if (r >= a.R) return;
    const Row<T> row(static_cast<const T *>(a.logits) + r * a.ld, a.V);
    T *out = static_cast<T *>(a.dlogits) + r * a.lddl;
    const int G = row.granules();
    TeacherShared &teacher = sh.teacher[TEACHER ? warp : 0];
    uint4 raw[U];
    const Step<T, 32, U> step(row, 0, lane, G);
    step.load(raw);
    int token = -1;
    float token_x = 0.f, mi = neg_inf(), si = 0.f;
    if constexpr (TEACHER) {
        Entries<T, 32> entries(a, r, lane);
        for (int i = lane; i < U * Elem<T>::kVec; i += 32) sh.bitmap[warp][i] = 0;
        if (lane == 0) teacher.bad = teacher.twice = 0;
        __syncwarp();
        entries.place(teacher, a, r, 0, row.n, lane);
        __syncwarp();
        teacher_weights<TAIL>(teacher, a.K);
        const uint32_t marked = entries.mark(teacher, a.K, sh.bitmap[warp], row.first(0), G * Elem<T>::kVec, lane);
        entries.settle(teacher, a.K, lane);
        if (TAIL && GRAD != kGradSaved) entries.add_marked(marked, a.c, mi, si);
        __syncwarp();
        if (TAIL && GRAD != kGradSaved) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t bits = u * 32 + lane < G ? bits_of<T>(sh.bitmap[warp], u * 32 + lane) : 0u;
                if (bits) raw[u] = without<T>(raw[u], bits);
            }
        }
    } else if (a.ids) {
        token = token_at(a, r);
        if (token >= 0 && token < a.V) token_x = Elem<T>::to_float(row.p[token]);
    }
    RowGrad k;
    if (GRAD != kGradSaved) {
        Running run = {neg_inf(), 0.f, 0.f};
        float all = Elem<T>::max_of(raw[0]);
#pragma unroll
        for (int u = 1; u < U; ++u) all = fmaxf(all, Elem<T>::max_of(raw[u]));
        raise<ENT>(run, all, a.c);
        accumulate<T, U, ENT>(raw, a.c, run);
        const Stats st = warp_stats<ENT, TAIL>(run, mi, si, a.c);
        const RowEnd e = row_end<TAIL>(st, a.c);
        if (lane == 0) write_sums<ENT, TAIL>(a, r, st, e, token, token_x);
        if (TEACHER && a.loss) {
            const float loss = teacher_loss<TAIL>(teacher, e, a.inv_t, a.K);
            if (lane == 0) a.loss[r] = loss;
        }
        if (MODE == kLogprobsTop) {
            const uint64_t *cand = sh.top[warp].cand;
            const int n = warp_top<T, U>(raw, row, G, a.K, sh.top[warp]);
            for (int i = lane; i < n; i += 32) {
                const uint64_t key = cand[i];
                int rank = 0;
#pragma unroll 4
                for (int j = 0; j < n; ++j) rank += cand[j] > key;
                if (rank >= a.K) continue;
                a.top_ids[r * a.K + rank] = static_cast<int32_t>(~static_cast<uint32_t>(key));
                a.top_logprobs[r * a.K + rank] = log_prob(unordered(static_cast<uint32_t>(key >> 32)), e, a.inv_t);
            }
        }
        if (GRAD == kNoGrad) return;
        k = TEACHER ? teacher_gradient<TAIL>(a, r, e, teacher) : token_gradient(a, r, st, e, token);
    } else {
        k = TEACHER ? teacher_gradient_saved<TAIL>(a, r, teacher) : token_gradient_saved(a, r, token);
    }
    // the elements are unpacked again rather than kept unpacked in twice the registers
#pragma unroll
    for (int u = 0; u < U; ++u) asm volatile("" : "+r"(raw[u].x), "+r"(raw[u].y), "+r"(raw[u].z), "+r"(raw[u].w));
    const Factors factors(k, a.c);
    constexpr bool SAVED = GRAD == kGradSaved;
    GradientWriter<T, ENT, SAVED>(row, out, factors).write(step, raw, a.c);
    __syncwarp();
    if (TEACHER) write_set_gradient<T, SAVED>(teacher, a.K, out, 0, row.n, a.c, k, lane, 32);
    else if (lane == 0 && token >= 0 && token < a.V) write_token_gradient<T, SAVED>(out, token, token_x, a.c, k);
}

// ------------------------------------------------------------------------------------------ long rows: a block or cluster each
__host__ __device__ constexpr int bitmap_words(int threads) { return threads == 128 ? 512 : 4096; }  // ids of one segment of a row, a bit each: all of a row for 128 threads, 2^17 for 256
constexpr int kGroupSteps = 32;     // groups a thread notes at most
// Threads a multiprocessor holds of the long rows' kernels.  With the ring 64 registers a thread are enough (16384 x 8192 bf16,
// distillation with gradient: 203 us with 768 threads, 186 with 1024); a step ahead in registers takes up to 80.  Blocks of 128
// where alternatives are looked for: 2048 x 131072 with the best 20 took 133 us with 256 threads, 125 with 128.
__host__ __device__ constexpr bool in_ring(int mode, int grad) { return mode >= kDistill || grad; }
__host__ __device__ constexpr int row_threads(int mode, int grad) { return in_ring(mode, grad) ? 1024 : 768; }

// Shared memory of a block beside the ring, and the steps of U granules a thread that its ring holds: what fits the multiprocessor's share, at most 4.
__host__ __device__ constexpr int fixed_shared(int mode, int threads) { return mode < kDistill ? 0 : static_cast<int>(sizeof(TeacherShared)) + (mode == kDistillTail ? 4 * bitmap_words(threads) : 0); }
__host__ __device__ constexpr int ring_steps(int mode, int grad, int threads, int u)
{
    return (227 * 1024 / (row_threads(mode, grad) / threads) - 2048 - fixed_shared(mode, threads)) / (16 * threads * u) < 4
               ? (227 * 1024 / (row_threads(mode, grad) / threads) - 2048 - fixed_shared(mode, threads)) / (16 * threads * u)
               : 4;
}

template <int NT> struct RowShared {
    Stats part[NT / 32];
    Stats pub;       // this block's sums, read by the cluster's other blocks
    RowEnd end;      // the row's
    RowGrad grad;
    Factors factors;
    uint32_t found;  // entries of top.best
};

// A row belongs to one block, or to a cluster whose blocks divide its granules.  A block's part goes through a ring of H steps in shared
// memory, each thread's granules copied by itself (so that no barrier is needed) up to H steps ahead.  With GRAD the row is then
// read again, backwards: its last H steps are still in the ring, the earlier ones in L2 as long as the rows in flight fit (see
// row_cluster).  A step ahead in registers instead took 246 us for 4096 x 65536 bf16 with gradient (now 214), and 136 for the
// distillation's loss alone (now 106); but the plain log probabilities, with the fewest instructions, lose to the way through shared memory
// (2048 x 131072: 99 us in registers, 105 through the ring), and where alternatives are looked for, these need the space.
// One row per block: with blocks that stay and walk over rows 8192 x 30000 with gradient took 236 us, now 211.
template <class T, int NT, int U, int MODE, int GRAD>
__global__ void __launch_bounds__(NT, row_threads(MODE, GRAD) / NT) loss_row_kernel(const LossArgs a)
{
    constexpr bool ENT = MODE == kLogprobs || MODE == kLogprobsTop, TOP = MODE == kLogprobsTop;
    constexpr bool TEACHER = MODE >= kDistill, TAIL = MODE == kDistillTail;
    constexpr int NW = NT / 32, STEP = NT * U;
    constexpr bool RING = in_ring(MODE, GRAD);
    constexpr int H = !RING ? 1 : ring_steps(MODE, GRAD, NT, U);
    extern __shared__ __align__(16) unsigned char dynamic[];
    __shared__ __align__(16) unsigned char shared_bytes[sizeof(RowShared<NT>)];
    RowShared<NT> &sh = *reinterpret_cast<RowShared<NT> *>(shared_bytes);
    TopShared &top = *reinterpret_cast<TopShared *>(dynamic);                               // TOP
    float *groups = reinterpret_cast<float *>(dynamic + sizeof(TopShared));                 // TOP
    TeacherShared &teacher = *reinterpret_cast<TeacherShared *>(dynamic);                   // TEACHER
    uint32_t *bitmap = reinterpret_cast<uint32_t *>(dynamic + sizeof(TeacherShared));       // TAIL

    cg::cluster_group cluster = cg::this_cluster();
    const int C = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t r = static_cast<int64_t>(blockIdx.x) / C;
    const int steps = a.steps;  // all rows take as many, some of the last granules may lie behind the row
    const Row<T> row(static_cast<const T *>(a.logits) + r * a.ld, a.V);
    const int g0 = min(row.granules(), rank * a.per_block), g1 = min(row.granules(), g0 + a.per_block);
    // without the ring: a step ahead in registers
    uint4 next[U];
    // with it: `slots` of the ring in use, `slot` the present one
    uint4 *const ring = reinterpret_cast<uint4 *>(dynamic + fixed_shared(MODE, NT)) + tid;
    const int slots = min(H, steps);
    int slot = 0;
    const auto fetch = [&](int step, int to) { Step<T, NT, U>(row, g0 + step * STEP, tid, g1).copy(ring + to * STEP); };
    // the present step's granules; the slots - 1 groups committed since are left on their way
    const auto take = [&](uint4 *to) {
        if (slots == 1) copies_wait<0>();
        else if (slots == 2) copies_wait<1>();
        else if (slots == 3) copies_wait<2>();
        else copies_wait<3>();
#pragma unroll
        for (int u = 0; u < U; ++u) to[u] = ring[slot * STEP + u * NT];
    };
    if (!RING) {
        Step<T, NT, U>(row, g0, tid, g1).load(next);
    } else {
        for (int i = 0; i < slots; ++i) {
            fetch(i, i);
            copies_commit();
        }
    }
    if (TAIL) {
        const int words = min(bitmap_words(NT), (steps * STEP * Elem<T>::kVec + 31) / 32);
        for (int i = tid; i < words; i += NT) bitmap[i] = 0;
    }
    Running run = {neg_inf(), 0.f, 0.f};
    float mi = neg_inf(), si = 0.f;
    int token = -1;
    float token_x = 0.f;
    uint32_t marked = 0;
    typename std::conditional<TEACHER, Entries<T, NT>, NoEntries>::type entries(a, r, tid);
    if constexpr (TEACHER) {
        if (tid == 0) teacher.bad = 0, teacher.twice = !TAIL;
        __syncthreads();
        entries.place_ids(teacher, a, tid);
        __syncthreads();
        if (warp == 0 && (rank == 0 || GRAD)) teacher_weights<TAIL>(teacher, a.K);
    } else if (a.ids) {
        token = token_at(a, r);
        if (token >= 0 && token < a.V && tid == 0) token_x = Elem<T>::to_float(row.p[token]);
    }

    constexpr int kSegment = bitmap_words(NT) * 32 / Elem<T>::kVec;  // granules
    static_assert(kSegment % STEP == 0, "a segment is whole steps");
    int shift = 0;
    if (TOP)
        while (steps >> shift >= kGroupSteps) ++shift;
    int step = 0;

    const int end = g0 + steps * STEP;
    for (int seg = g0; seg < end; seg = TAIL ? seg + kSegment : end) {
        const int seg_end = TAIL ? min(end, seg + kSegment) : end;
        if constexpr (TAIL) {
            const uint32_t now = entries.mark(teacher, a.K, bitmap, row.first(seg), (min(seg_end, g1) - seg) * Elem<T>::kVec, tid);
            marked |= now;
            __syncthreads();
        }
        for (int base = seg; base < seg_end; base += STEP, ++step) {
            uint4 cur[U];
            if (!RING) {
#pragma unroll
                for (int u = 0; u < U; ++u) cur[u] = next[u];
                if (step + 1 < steps) Step<T, NT, U>(row, base + STEP, tid, g1).load(next);
            } else {
                take(cur);
            }
            if (TAIL) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const uint32_t bits = bits_of<T>(bitmap, base + u * NT + tid - seg);
                    if (bits) cur[u] = without<T>(cur[u], bits);
                }
            }
            float all = Elem<T>::max_of(cur[0]);
#pragma unroll
            for (int u = 1; u < U; ++u) all = fmaxf(all, Elem<T>::max_of(cur[u]));
            if (TOP) {
                float *slot = groups + (step >> shift) * NT + tid;
                const float largest = base + tid < g1 ? all : quiet_nan();
                *slot = step & ((1 << shift) - 1) ? fmaxf(largest, *slot) : largest;
            }
            raise<ENT>(run, all, a.c);
            accumulate<T, U, ENT>(cur, a.c, run);
            if (RING) {
                if (step + slots < steps) fetch(step + slots, slot);
                copies_commit();
                slot = slot + 1 == slots ? 0 : slot + 1;
            }
        }
        if constexpr (TAIL) {
            if (seg_end == end) break;
            __syncthreads();
            entries.unmark(teacher, a.K, bitmap, row.first(seg), (min(seg_end, g1) - seg) * Elem<T>::kVec, tid);
            __syncthreads();
        }
    }

    if constexpr (TEACHER) {
        entries.gather(teacher, a.K, row.p, rank == 0 ? 0 : row.first(g0), rank == 0 ? row.n : row.first(g1), tid);
        if constexpr (TAIL) entries.add_marked(marked, a.c, mi, si);
        entries.settle(teacher, a.K, tid);
    }
    Stats st = warp_stats<ENT, TAIL>(run, mi, si, a.c);
    if (lane == 0) sh.part[warp] = st;
    __syncthreads();
    // The first warp alone joins the sums and works out what the row needs; a row's other threads only read the factors.
    if (warp == 0) {
        st = lane < NW ? sh.part[lane] : Stats{neg_inf(), 0.f, 0.f, neg_inf(), 0.f};
#pragma unroll
        for (int d = NW / 2; d; d >>= 1) join_stats<ENT, TAIL>(st, shuffle_xor<ENT, TAIL>(st, d), a.c);
        if (C > 1 && lane == 0) sh.pub = st;
    }
    if (TOP) {
        const int e0 = max(0, row.first(g0)), e1 = min(row.n, row.first(g1));
        const int want = max(0, min(a.K, e1 - e0));
        if (want > 0) find_top<T, NT, U>(top, groups, (steps + (1 << shift) - 1) >> shift, shift, row, g0, g1, want);
        if (tid == 0) sh.found = static_cast<uint32_t>(want);
    }
    if (C > 1) {
        cluster.sync();
        if (warp == 0 && (rank == 0 || GRAD)) {
            st = lane < C ? *cluster.map_shared_rank(&sh.pub, lane) : Stats{neg_inf(), 0.f, 0.f, neg_inf(), 0.f};
#pragma unroll
            for (int d = 4; d; d >>= 1) join_stats<ENT, TAIL>(st, shuffle_xor<ENT, TAIL>(st, d), a.c);
        }
        if (TOP && rank == 0) {
            int n = 0;  // the blocks' lists side by side
            for (int b = 0; b < C; ++b) {
                const int m = static_cast<int>(*cluster.map_shared_rank(&sh.found, b));
                const TopShared *other = cluster.map_shared_rank(&top, b);
                for (int i = tid; i < m; i += NT) top.cand[n + i] = other->best[i];
                n += m;
            }
        }
        cluster.barrier_arrive();  // its other half stands at the row's end: shared memory may be read until then
        if (TOP && rank == 0) {
            __syncthreads();
            int n = 0;
            for (int b = 0; b < C; ++b) n += share_count<T>(row, a.per_block, b, a.K);
            select_top<NT>(top, n, a.K);
        }
    }
    if (warp == 0 && (rank == 0 || GRAD)) {
        const RowEnd e = row_end<TAIL>(st, a.c);
        if (GRAD) {
            const RowGrad k = TEACHER ? teacher_gradient<TAIL>(a, r, e, teacher) : token_gradient(a, r, st, e, token);
            const Factors f(k, a.c);
            if (lane == 0) sh.grad = k, sh.factors = f;
        }
        if (lane == 0) sh.end = e;
        if (lane == 0 && rank == 0) write_sums<ENT, TAIL>(a, r, st, e, token, token_x);
    }
    if (GRAD || TEACHER || TOP) __syncthreads();
    if (rank == 0) {
        if (TEACHER && warp == NW - 1 && a.loss) {
            const float loss = teacher_loss<TAIL>(teacher, sh.end, a.inv_t, a.K);
            if (lane == 0) a.loss[r] = loss;
        }
        if (TOP) {
            for (int i = tid; i < a.K; i += NT) {
                const uint64_t key = top.best[i];
                a.top_ids[r * a.K + i] = static_cast<int32_t>(~static_cast<uint32_t>(key));
                a.top_logprobs[r * a.K + i] = log_prob(unordered(static_cast<uint32_t>(key >> 32)), sh.end, a.inv_t);
            }
        }
    }
    if (GRAD) {
        T *out = static_cast<T *>(a.dlogits) + r * a.lddl;
        const GradientWriter<T, ENT, false> writer(row, out, sh.factors);
        for (step = steps - 1; step >= 0; --step) {
            uint4 cur[U];
            slot = slot == 0 ? slots - 1 : slot - 1;
            take(cur);
            writer.write(Step<T, NT, U>(row, g0 + step * STEP, tid, g1), cur, a.c);
            if (step >= slots) fetch(step - slots, slot);
            copies_commit();
        }
        __syncthreads();
        if (TEACHER) write_set_gradient<T, false>(teacher, a.K, out, row.first(g0), row.first(g1), a.c, sh.grad, tid, NT);
        else if (tid == 0 && token >= 0 && token < a.V && token >= row.first(g0) && token < row.first(g1)) write_token_gradient<T, false>(out, token, token_x, a.c, sh.grad);
    }
    if (C > 1) cluster.barrier_wait();
}

// Gradients from saved sums: one read and one write of the row, a.segments blocks per row (it needs nothing of the row's other
// parts), the next U granules of a thread in flight while the present ones are written.  Bound by memory and the issue slots alike.
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
    RowGrad k;
    int token = -1;
    float token_x = 0.f;
    uint4 next[U];
    typename std::conditional<TEACHER, Entries<T, NT>, NoEntries>::type entries(a, r, threadIdx.x);
    Step<T, NT, U>(row, g0, threadIdx.x, g1).load_again(next);
    if constexpr (TEACHER) {
        if (threadIdx.x == 0) shared.bad = 0, shared.twice = 1;
        __syncthreads();
        entries.place(shared, a, r, row.first(g0), row.first(g1), threadIdx.x);
        __syncthreads();
        if (threadIdx.x < 32) teacher_weights<TAIL>(shared, a.K);
        __syncthreads();
        k = teacher_gradient_saved<TAIL>(a, r, shared);
    } else {
        if (a.grad) token = token_at(a, r);
        k = token_gradient_saved(a, r, token);
        if (token < row.first(g0) || token >= row.first(g1) || token >= a.V) token = -1;  // another block's, or none
        if (threadIdx.x == 0 && token >= 0) token_x = Elem<T>::to_float(row.p[token]);
        __syncthreads();  // read before it is overwritten in place
    }
    const Factors factors(k, a.c);
    const GradientWriter<T, !TEACHER, true> writer(row, out, factors);
    for (int base = g0; base < g1; base += NT * U) {
        uint4 cur[U];
#pragma unroll
        for (int u = 0; u < U; ++u) cur[u] = next[u];
        if (base + NT * U < g1) Step<T, NT, U>(row, base + NT * U, threadIdx.x, g1).load_again(next);
        writer.write(Step<T, NT, U>(row, base, threadIdx.x, g1), cur, a.c);
    }
    if constexpr (TEACHER) entries.settle(shared, a.K, threadIdx.x);
    __syncthreads();
    if constexpr (TEACHER) write_set_gradient<T, true>(shared, a.K, out, row.first(g0), row.first(g1), a.c, k, threadIdx.x, NT);
    else if (threadIdx.x == 0 && token >= 0) write_token_gradient<T, true>(out, token, token_x, a.c, k);
}

// ------------------------------------------------------------------------------------------ launches
// Granules of the logits' longest row: one more where rows do not start on 16 bytes.
template <class T> inline int64_t most_granules(const LossArgs &a)
{
    return (a.V + Elem<T>::kVec - 1) / Elem<T>::kVec + (aligned(a.logits, 16) && a.ld % Elem<T>::kVec == 0 ? 0 : 1);
}

constexpr int64_t kMostBlocks = 0x7fffffff;
constexpr int64_t kL2 = 64;  // MB
constexpr int kSteps = 4;  // granules per thread and step of the long rows' kernels

template <class T, int NT, int MODE, int GRAD> inline int launch_row(LossArgs a, int cluster, cudaStream_t stream)
{
    if (a.R > kMostBlocks / cluster) return SPDY_ERR_UNSUPPORTED;
    auto *kernel = loss_row_kernel<T, NT, kSteps, MODE, GRAD>;
    constexpr int kStep = NT * kSteps;
    a.per_block = static_cast<int>((most_granules<T>(a) + cluster - 1) / cluster);
    a.steps = (a.per_block - 1) / kStep + 1;
    size_t smem = 0;
    if (in_ring(MODE, GRAD)) {
        constexpr int H = ring_steps(MODE, GRAD, NT, kSteps);
        static_assert(!in_ring(MODE, GRAD) || H >= 2, "");
        smem = fixed_shared(MODE, NT) + 16 * kStep * static_cast<size_t>(std::min(H, a.steps));
        if (smem > 40 * 1024) SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    } else if (MODE == kLogprobsTop) {
        smem = sizeof(TopShared) + sizeof(uint32_t) * NT * static_cast<size_t>(std::min(a.steps, kGroupSteps));
        SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           static_cast<int>(sizeof(TopShared) + sizeof(uint32_t) * NT * kGroupSteps)));
    }
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>(a.R * cluster));
    config.blockDim = dim3(NT);
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

// Blocks that share a row (a cluster, its sums exchanged through the blocks' shared memory): more when the rows alone would not
// fill the device twice and every block still has a step of work; with a gradient also as many as keep what the ring does not hold
// of the rows in flight within 64 MB of L2.  No more than that to fill the last round of rows (two blocks to a row: 640 x 32768
// f16, distillation with gradient 24.7 to 28.8 us).  (2048 x 131072 bf16, distillation with gradient: one block to a row 235 us, two 222,
// four 248).
template <class T, int NT, int MODE, int GRAD> inline int row_cluster(const LossArgs &a)
{
    const int64_t G = most_granules<T>(a), slots = static_cast<int64_t>(sm_count()) * (row_threads(MODE, GRAD) / NT);
    int cluster = 1;
    if (GRAD)
        while (cluster < 8 && slots * 16 * (G / cluster - ring_steps(MODE, GRAD, NT, kSteps) * NT * kSteps) > (kL2 << 20)) cluster *= 2;
    while (cluster < 8 && a.R * cluster < 2 * sm_count() && G > static_cast<int64_t>(cluster) * NT * kSteps) cluster *= 2;
    return cluster;
}

template <class T, int U, int MODE, int GRAD> inline int launch_warp(const LossArgs &a, cudaStream_t stream)
{
    const int64_t blocks = (a.R + kWarpRows - 1) / kWarpRows;
    if (blocks > kMostBlocks) return SPDY_ERR_UNSUPPORTED;
    loss_warp_kernel<T, U, MODE, GRAD><<<static_cast<unsigned>(blocks), 32 * kWarpRows, 0, stream>>>(a);
    return finish_launch();
}

// The forward pass, with the gradient too where GRAD says so.
template <class T, int MODE, int GRAD> int rows(const LossArgs &a, cudaStream_t stream)
{
    const int64_t G = most_granules<T>(a);
    if (G <= 128) return launch_warp<T, 4, MODE, GRAD>(a, stream);
    if (G <= 256) return launch_warp<T, 8, MODE, GRAD>(a, stream);
    // blocks of 128 up to 1024 granules: 16384 x 8000 bf16 82 us, with 256 threads 117
    if constexpr (MODE == kLogprobsTop) return launch_row<T, 128, MODE, GRAD>(a, row_cluster<T, 128, MODE, GRAD>(a), stream);
    else if (G <= 1024) return launch_row<T, 128, MODE, GRAD>(a, row_cluster<T, 128, MODE, GRAD>(a), stream);
    else return launch_row<T, 256, MODE, GRAD>(a, row_cluster<T, 256, MODE, GRAD>(a), stream);
}

template <class T, int MODE, int NT> int backward_rows(LossArgs a, int64_t G, cudaStream_t stream)
{
    constexpr int U = kSteps;
    a.segments = static_cast<int>((G + 2 * NT * U - 1) / (2 * NT * U));
    if (a.R * a.segments < 4 * sm_count()) a.segments = static_cast<int>((G + NT - 1) / NT);
    if (a.R * a.segments > kMostBlocks) return SPDY_ERR_UNSUPPORTED;
    loss_backward_kernel<T, NT, U, MODE >= kDistill, MODE == kDistillTail><<<static_cast<unsigned>(a.R * a.segments), NT, 0, stream>>>(a);
    return finish_launch();
}
template <class T, int MODE> int backward(const LossArgs &a, cudaStream_t stream)
{
    const int64_t G = most_granules<T>(a);
    if (G <= 128) return launch_warp<T, 4, MODE, kGradSaved>(a, stream);
    if (G <= 256) return launch_warp<T, 8, MODE, kGradSaved>(a, stream);
    // as for the forward pass; 16384 x 2300 bf16: 48 us, with 256 threads 85
    return G <= 1024 ? backward_rows<T, MODE, 128>(a, G, stream) : backward_rows<T, MODE, 256>(a, G, stream);
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
