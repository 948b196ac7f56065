// Shared by the evaluation operators (eval_*.cu): element types, 16-byte granules of rows that start anywhere, running
// softmax sums, launch helpers.
#ifndef SPDY_EVAL_COMMON_CUH
#define SPDY_EVAL_COMMON_CUH

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/spdy_eval.h"
#include "eval_ranges.h"

namespace spdy {
void note_cuda_error(int err);  // spdy_api.cu: what spdy_last_cuda_error() reports
}

namespace spdy_eval {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// 2^x on the special-function unit; results below 2^-126 become 0, which is what a softmax term that small adds.
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// max(a, b) and min(a, b) that keep NaN (fmaxf and fminf drop it).
__device__ __forceinline__ float max_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

__device__ __forceinline__ float min_nan(float a, float b)
{
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float quiet_nan() { return __int_as_float(0x7fc00000); }

__device__ __forceinline__ uint4 load_stream(const void *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Read for the last time, or written to be read much later: first to leave L2 (the streaming forms need no policy register;
// with an explicit one each access cost two more instructions).
__device__ __forceinline__ uint4 load_last(const void *p)
{
    uint4 v;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void store_last(void *p, uint4 v)
{
    asm volatile("st.global.cs.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void store_stream(void *p, uint4 v)
{
    asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// 16 bytes to shared memory, both ends aligned; counted by commit and waited for by the issuing thread.
__device__ __forceinline__ void copy16(void *to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(to))), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until at most N of the thread's groups of copies are on their way.
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Element types: how many fit 16 bytes, conversion, and the bit pattern of -inf repeated over a word.
template <class T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kVec = 4;
    static constexpr uint32_t kNegInfWord = 0xff800000u;
    static __device__ __forceinline__ float to_float(float x) { return x; }
    static __device__ __forceinline__ float from_float(float x) { return x; }
    static __device__ __forceinline__ void unpack(uint4 r, float *f)
    {
        f[0] = __uint_as_float(r.x), f[1] = __uint_as_float(r.y), f[2] = __uint_as_float(r.z), f[3] = __uint_as_float(r.w);
    }
    static __device__ __forceinline__ uint4 pack(const float *f)
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    // largest of the granule, NaN left aside (NaN only if there is nothing else)
    static __device__ __forceinline__ float max_of(uint4 r)
    {
        return fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w)));
    }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int kVec = 8;
    static constexpr uint32_t kNegInfWord = 0xff80ff80u;
    static __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
    static __device__ __forceinline__ void two(uint32_t w, float &lo, float &hi)
    {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xffff0000u);
    }
    static __device__ __forceinline__ void unpack(uint4 r, float *f)
    {
        two(r.x, f[0], f[1]), two(r.y, f[2], f[3]), two(r.z, f[4], f[5]), two(r.w, f[6], f[7]);
    }
    static __device__ __forceinline__ uint32_t join(float lo, float hi)
    {
        __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t *>(&v);
    }
    static __device__ __forceinline__ uint4 pack(const float *f) { return make_uint4(join(f[0], f[1]), join(f[2], f[3]), join(f[4], f[5]), join(f[6], f[7])); }
    static __device__ __forceinline__ float max_of(uint4 r)
    {
        const __nv_bfloat162 *h = reinterpret_cast<const __nv_bfloat162 *>(&r);
        const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
};
template <> struct Elem<__half> {
    static constexpr int kVec = 8;
    static constexpr uint32_t kNegInfWord = 0xfc00fc00u;
    static __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }
    static __device__ __forceinline__ void two(uint32_t w, float &lo, float &hi)
    {
        const float2 v = __half22float2(*reinterpret_cast<__half2 *>(&w));
        lo = v.x, hi = v.y;
    }
    static __device__ __forceinline__ void unpack(uint4 r, float *f)
    {
        two(r.x, f[0], f[1]), two(r.y, f[2], f[3]), two(r.z, f[4], f[5]), two(r.w, f[6], f[7]);
    }
    static __device__ __forceinline__ uint32_t join(float lo, float hi)
    {
        __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t *>(&v);
    }
    static __device__ __forceinline__ uint4 pack(const float *f) { return make_uint4(join(f[0], f[1]), join(f[2], f[3]), join(f[4], f[5]), join(f[6], f[7])); }
    static __device__ __forceinline__ float max_of(uint4 r)
    {
        const __half2 *h = reinterpret_cast<const __half2 *>(&r);
        const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
};

// Granules that lie only partly inside a row of n elements, from element e (of row p or q) on: kept out of line, they are few.
template <class T> __device__ __noinline__ uint4 load_part(const T *p, int n, int e)
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j, e += 4 / static_cast<int>(sizeof(T))) {
        w[j] = Elem<T>::kNegInfWord;
        if (sizeof(T) == 4) {
            if (e >= 0 && e < n) w[j] = reinterpret_cast<const uint32_t *>(p)[e];
        } else {
            if (e >= 0 && e < n) w[j] = (w[j] & 0xffff0000u) | reinterpret_cast<const uint16_t *>(p)[e];
            if (e + 1 >= 0 && e + 1 < n) w[j] = (w[j] & 0xffffu) | static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[e + 1]) << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <class T> __device__ __noinline__ void store_part(T *q, int n, int e, uint4 v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j, e += 4 / static_cast<int>(sizeof(T))) {
        if (sizeof(T) == 4) {
            if (e >= 0 && e < n) reinterpret_cast<uint32_t *>(q)[e] = w[j];
        } else {
            if (e >= 0 && e < n) reinterpret_cast<uint16_t *>(q)[e] = static_cast<uint16_t>(w[j]);
            if (e + 1 >= 0 && e + 1 < n) reinterpret_cast<uint16_t *>(q)[e + 1] = static_cast<uint16_t>(w[j] >> 16);
        }
    }
}

// A row that may start anywhere: granule g is the g-th aligned 16 bytes that hold a part of it, elements
// g * kVec - lead .. + kVec - 1.  Only granules that lie wholly inside the row are moved 16 bytes at a time.
template <class T> struct Row {
    const T *p;
    int n;       // elements, at most 2^31 - 65 (positions inside a row are 32-bit)
    int lead;    // elements of granule 0 that lie before the row

    __device__ __forceinline__ Row(const T *row, int64_t count) : p(row), n(static_cast<int>(count)), lead(static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T))) {}
    __device__ __forceinline__ int granules() const { return (n + lead + Elem<T>::kVec - 1) / Elem<T>::kVec; }
    __device__ __forceinline__ int first(int g) const { return g * Elem<T>::kVec - lead; }
    __device__ __forceinline__ bool whole(int g) const { return first(g) >= 0 && first(g) <= n - Elem<T>::kVec; }
    // elements outside the row read as -inf
    __device__ __forceinline__ uint4 load(int g) const
    {
        if (whole(g)) return load_stream(p + first(g));
        return load_part(p, n, first(g));
    }
    // granules g0 .. g1 - 1 are all whole
    __device__ __forceinline__ bool inner(int g0, int g1) const { return first(g0) >= 0 && first(g1) <= n; }
    __device__ __forceinline__ bool same_lead(const T *q) const { return (reinterpret_cast<uintptr_t>(q) & 15) == (reinterpret_cast<uintptr_t>(p) & 15); }
};

// The granules base + t, base + t + NT, ... (U of them) of a row, for a block or warp of NT threads: where all are whole and
// below `limit`, one test serves them all; else each is tested, and reads as -inf from granule `limit` on.
template <class T, int NT, int U> struct Step {
    const Row<T> &row;
    int g, limit;
    bool plain;
    __device__ __forceinline__ Step(const Row<T> &r, int base, int t, int limit_) : row(r), g(base + t), limit(limit_)
    {
        plain = base + NT * U <= limit_ && r.inner(base, base + NT * U);
    }
    __device__ __forceinline__ uint4 load_part_of(int u) const
    {
        constexpr uint32_t NI = Elem<T>::kNegInfWord;
        const int at = g + u * NT;
        if (at >= limit) return make_uint4(NI, NI, NI, NI);
        return row.whole(at) ? load_stream(row.p + row.first(at)) : load_part(row.p, row.n, row.first(at));
    }
    __device__ __forceinline__ void load(uint4 *v) const
    {
        if (plain) {
            const T *p = row.p + row.first(g);
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_stream(p + u * NT * Elem<T>::kVec);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_part_of(u);
        }
    }
    // to shared memory, granule u to to[u * NT]; asynchronous but for the row's ends
    __device__ __forceinline__ void copy(uint4 *to) const
    {
        constexpr uint32_t NI = Elem<T>::kNegInfWord;
        if (plain) {
            const T *p = row.p + row.first(g);
#pragma unroll
            for (int u = 0; u < U; ++u) copy16(to + u * NT, p + u * NT * Elem<T>::kVec);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = g + u * NT;
                if (at >= limit) to[u * NT] = make_uint4(NI, NI, NI, NI);
                else if (row.whole(at)) copy16(to + u * NT, row.p + row.first(at));
                else to[u * NT] = load_part(row.p, row.n, row.first(at));
            }
        }
    }
    __device__ __forceinline__ void load_again(uint4 *v) const  // not to be read after this
    {
        if (plain) {
            const T *p = row.p + row.first(g);
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_last(p + u * NT * Elem<T>::kVec);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load_part_of(u);
        }
    }
    // to granule u of `q`, a row of as many elements that may start elsewhere (`same`: it does not)
    __device__ __forceinline__ void store_part_of(T *q, bool same, int u, uint4 v) const
    {
        const int at = g + u * NT;
        if (at >= limit) return;
        if (same && row.whole(at)) store_stream(q + row.first(at), v);
        else store_part(q, row.n, row.first(at), v);
    }
};

// Sums of exponentials relative to a running maximum: s = sum 2^((x - m) c) over some logits x, c = log2(e) / T > 0.  The
// maximum is kept unscaled, so that logits near the largest finite numbers (masks of the type's lowest value) do not
// overflow; the empty sum is (-inf, 0).  A NaN or +inf among the logits makes s NaN.
__device__ __forceinline__ void join_sums(float &m, float &s, float om, float os, float c)
{
    const float top = fmaxf(m, om);
    if (s != 0.f) s *= ex2((m - top) * c);
    if (os != 0.f) s = fmaf(os, ex2((om - top) * c), s);
    m = top;
}
__device__ __forceinline__ void add_logit(float &m, float &s, float x, float c)
{
    if (x != neg_inf()) join_sums(m, s, x, x - x + 1.f, c);
}

inline bool known_type(int t) { return t == SPDY_F32 || t == SPDY_BF16 || t == SPDY_F16; }
inline size_t type_size(int t) { return t == SPDY_F32 ? 4 : 2; }
inline bool temperature_ok(float t) { return t > 0.f && t <= 3.4e38f && kLog2e / t <= 3.4e38f && kLog2e / t > 0.f; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int finish_launch()
{
    const cudaError_t err = cudaGetLastError();
    if (err == cudaSuccess) return SPDY_OK;
    spdy::note_cuda_error(static_cast<int>(err));
    return SPDY_ERR_CUDA;
}

#define SPDY_EVAL_TRY(expr)                                    \
    do {                                                       \
        const cudaError_t err__ = (expr);                      \
        if (err__ != cudaSuccess) {                            \
            (void)cudaGetLastError();                          \
            spdy::note_cuda_error(static_cast<int>(err__));    \
            return SPDY_ERR_CUDA;                              \
        }                                                      \
    } while (0)

// Multiprocessors of the current device (asked once per device).
int sm_count();

}  // namespace spdy_eval
#endif
