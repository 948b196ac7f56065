// AdamW steps over many tensors at once, with moments in 32 or in 8 bits: kernels and C entries (spdy_eval.h).
//
//   g = grad * grad_scale,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   param = param (1 - lr weight_decay) - lr / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
//
// Moments in 8 bits: 32 consecutive elements share a byte E, the fp32 exponent field (at least 1) of the largest magnitude among
// them; an element y is a small floating-point number relative to 2^(E - 127), and fp32's own layout does the conversion: times a
// power of two that puts the block's largest into exponent field 14 (first moment: sign, 4 bits of exponent, 3 of mantissa) or 30
// (second: 5 and 3), the upper bits of y's pattern ARE the code, its lower 20 bits the part cut off, fields of 0 included, since fp32
// has them too.  20 random bits added before the cut round it up with the right probability: an average that moves by 1 - beta2 = 0.1 %
// of itself a step would stand still under rounding to nearest, with steps of 6 to 12 %.  A positive second moment is never rounded to
// 0: its floor, 2^-32 of the block's largest, is what keeps m / sqrt(v) of small elements bounded (m itself ends at 2^-17).
// The random bits are a hash of (seed, step, tensor, element), so a step can be repeated bit for bit.
#include "eval_common.cuh"

using namespace spdy_eval;

namespace {

// A block works on 2048 elements at a time, a thread on 8 of them, or on 16 with moments in 8 bits, where what is done per thread
// (addresses, the tensor's entry, the blocks' exponents) weighs more than registers.
constexpr int kChunk = 2048, kBlock = 32;                          // kBlock: elements that share an exponent
template <int BITS> constexpr int kPer = BITS == 8 ? 16 : 8;
template <int BITS> constexpr int kThreads = kChunk / kPer<BITS>;

struct Entry {
    void *param;
    const void *grad;
    float *master;
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    int64_t n;
    uint32_t first;       // chunks of the tensors before it
    float weight_decay, decay;  // decay: 1 - lr weight_decay, where lr is known
    uint32_t index;       // in the caller's list
    uint32_t flags;
    uint32_t unused;
};
enum { kWide = 1, kWideStates = 2, kKeepZeros = 4 };  // kWide: param, grad and master start on 32 bytes; kWideStates: so do m and v

struct StepArgs {
    float b1, b2, g1, g2, eps, rate, root;  // g1 = 1 - b1, rate = lr / (1 - b1^t), root = 1 / sqrt(1 - b2^t)
    double lr, beta1, beta2;
    uint32_t seed, key;                     // key: of seed and step
    const float *lr_device, *grad_scale, *skip;
    const int64_t *step_device;
};

// As many tensors as a launch's parameters (32764 bytes) hold; few of them for small calls, whose launch then copies less.
template <int CAP> struct Table {
    Entry e[CAP];
    uint32_t count, chunks;
};
constexpr int kFew = 16, kMany = 360;

// The tensor that a chunk belongs to.
template <int CAP> __device__ __forceinline__ uint32_t tensor_of(const Table<CAP> &table, uint32_t chunk)
{
    uint32_t low = 0, high = table.count;  // first[low] <= chunk < first[high]
    while (high - low > 1) {
        const uint32_t mid = (low + high) / 2;
        if (chunk >= table.e[mid].first) low = mid;
        else high = mid;
    }
    return low;
}

// A hash of 32 bits: "lowbias32", as Chris Wellons published it (two odd multipliers, each of which carries bits up, and shifts that bring them down
// again; the constants are the ones found there to leave the least bias).
SPDY_EVAL_FN uint32_t mix(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x7feb352du;
    x = (x ^ (x >> 15)) * 0x846ca68bu;
    return x ^ (x >> 16);
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float exponent(int field) { return __int_as_float(field << 23); }  // 2^(field - 127), 1 <= field <= 254

// The two formats: the exponent field that the largest magnitude's binade gets.
template <bool SIGNED> constexpr int kField = SIGNED ? 14 : 30;

// Eight numbers from their codes and the block's byte.  A code's bits, four below the top of a word, are the upper bits of a float
// whose exponent is off by a known amount: one product puts it right (two where 2^(E - 14) or 2^(E - 30) is no float).
template <bool SIGNED, int N> __device__ __forceinline__ void decode(const uint32_t *codes, uint32_t E, float *y)
{
    constexpr uint32_t most = 254 - 127 + kField<SIGNED>;  // the largest E whose factor is a float
    const float factor = E == 255 ? quiet_nan() : exponent(min(static_cast<int>(E), static_cast<int>(most)) + 127 - kField<SIGNED>);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t top = __byte_perm(codes[i / 4], 0, (i % 4) << 12 | 0x0444);  // the code in the highest byte
        y[i] = (SIGNED ? __uint_as_float(static_cast<uint32_t>(static_cast<int32_t>(top) >> 4) & 0x87f00000u) : __uint_as_float(top >> 4)) * factor;
    }
    if (E > most && E != 255)
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] *= exponent(127 + static_cast<int>(E - most));
}

// Codes of a thread's N elements (a part of a block, which neighbouring lanes share), and the block's byte.
template <bool SIGNED, int N> __device__ __forceinline__ void encode(float *y, const uint32_t *random, uint32_t *codes, uint32_t &E)
{
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) most = max_nan(most, fabsf(y[i]));
#pragma unroll
    for (int d = 1; d < kBlock / N; d *= 2) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, d));
    E = max(__float_as_uint(most) >> 23, 1u);
    const bool bad = E >= 254;
    int field = 127 + kField<SIGNED> - static_cast<int>(E);  // of the factor
    if (field < 1) {  // no float: the way down in two steps, of which the first is exact for all that is left after the second
        field += 113;
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = !SIGNED && y[i] > 0.f ? fmaxf(y[i] * 0x1p-113f, 0x1p-149f) : y[i] * 0x1p-113f;  // positive stays positive, for the floor below
    }
    if (bad) E = 255;
    const float factor = exponent(max(field, 1));
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        uint32_t x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t bits = __float_as_uint(fabsf(y[i + k]) * factor);
            if (SIGNED) {
                x[k] = (bits + (random[i + k] & 0xfffffu)) << 4 | (__float_as_uint(y[i + k]) & 0x80000000u);
            } else {  // the part of `random` below its upper 20 bits lies below the code's own last bit and carries nothing
                x[k] = (bits << 4) + (random[i + k] >> 8);
                if (y[i + k] > 0.f) x[k] = max(x[k], 1u << 24);
            }
        }
        codes[i / 4] = bad ? 0 : __byte_perm(__byte_perm(x[0], x[1], 0x0073), __byte_perm(x[2], x[3], 0x0073), 0x5410);
    }
}

// 16 bytes of a vector of which `left` elements exist, zeros for the others; and the way back.
template <class T> __device__ __noinline__ uint4 gather(const T *p, int left)
{
    constexpr int bits = 8 * sizeof(T), per = 32 / bits;
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        w[j] = 0;
#pragma unroll
        for (int k = 0; k < per; ++k) {
            const int i = j * per + k;
            uint32_t x = 0;
            if (i < left) x = bits == 32 ? reinterpret_cast<const uint32_t *>(p)[i] : bits == 16 ? reinterpret_cast<const uint16_t *>(p)[i] : reinterpret_cast<const uint8_t *>(p)[i];
            w[j] |= x << (bits * k & 31);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <class T> __device__ __noinline__ void scatter(T *p, int left, uint4 v)
{
    constexpr int bits = 8 * sizeof(T), per = 32 / bits;
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int k = 0; k < per; ++k) {
            const int i = j * per + k;
            if (i >= left) continue;
            const uint32_t x = w[j] >> (bits * k & 31);
            if (bits == 32) reinterpret_cast<uint32_t *>(p)[i] = x;
            else if (bits == 16) reinterpret_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(x);
            else reinterpret_cast<uint8_t *>(p)[i] = static_cast<uint8_t>(x);
        }
}
// 32 bytes, first to leave L2: everything is read once and written once (150 M elements with fp32 states and masters 653 us without that,
// 614 with it).
__device__ __forceinline__ void load_pair(const void *p, uint4 &lo, uint4 &hi)
{
    asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(lo.x), "=r"(lo.y), "=r"(lo.z), "=r"(lo.w), "=r"(hi.x), "=r"(hi.y), "=r"(hi.z), "=r"(hi.w)
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store_pair(void *p, uint4 lo, uint4 hi)
{
    asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(lo.x), "r"(lo.y), "r"(lo.z), "r"(lo.w), "r"(hi.x),
                 "r"(hi.y), "r"(hi.z), "r"(hi.w)
                 : "memory");
}
// N elements from `p` on; `whole`: all exist, and p lies on 32 bytes (16, where they are no more).
template <class T, int N> __device__ __forceinline__ void load(const T *p, int left, bool whole, uint4 *raw)
{
    constexpr int per = 16 / sizeof(T);
    if (whole) {
        if constexpr (N / per == 1) raw[0] = load_last(p);
        else
#pragma unroll
            for (int j = 0; j < N / per; j += 2) load_pair(p + j * per, raw[j], raw[j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < N / per; ++j) raw[j] = gather<T>(p + j * per, left - j * per);
    }
}
template <class T, int N> __device__ __forceinline__ void store(T *p, int left, bool whole, const uint4 *raw)
{
    constexpr int per = 16 / sizeof(T);
    if (whole) {
        if constexpr (N / per == 1) store_last(p, raw[0]);
        else
#pragma unroll
            for (int j = 0; j < N / per; j += 2) store_pair(p + j * per, raw[j], raw[j + 1]);
    } else {
#pragma unroll
        for (int j = 0; j < N / per; ++j) scatter<T>(p + j * per, left - j * per, raw[j]);
    }
}
template <class T, int N> __device__ __forceinline__ void unpack(const uint4 *raw, float *f)
{
#pragma unroll
    for (int j = 0; j < N / Elem<T>::kVec; ++j) Elem<T>::unpack(raw[j], f + j * Elem<T>::kVec);
}
template <class T, int N> __device__ __forceinline__ void pack(const float *f, uint4 *raw)
{
#pragma unroll
    for (int j = 0; j < N / Elem<T>::kVec; ++j) raw[j] = Elem<T>::pack(f + j * Elem<T>::kVec);
}

// y to 16 bits, up with the probability of the part cut off: fp32's pattern again, brought to half precision's exponents by a power of two.
template <class T> __device__ __forceinline__ uint32_t round_random(float y, uint32_t random)
{
    constexpr bool brain = std::is_same<T, __nv_bfloat16>::value;
    constexpr int shift = brain ? 16 : 13;
    const uint32_t sign = __float_as_uint(y) >> 16 & 0x8000u;
    const uint32_t code = (__float_as_uint(fabsf(y) * (brain ? 1.f : 0x1p-112f)) + (random >> (32 - shift))) >> shift;
    const uint32_t infinite = brain ? 0x7f80u : 0x7c00u;
    if (!(fabsf(y) <= 3.4028235e38f)) return y == y ? sign | infinite : 0x7fffu;  // a NaN in both
    return sign | min(code, infinite);
}
// N of them.  In bf16, finite numbers only need the addition: its carry ends at the exponent, and the sign stays above it.
template <class T, int N> __device__ __forceinline__ void pack_random(const float *y, const uint32_t *random, uint4 *raw)
{
    uint32_t w[N / 2];
    float odd = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) odd = fmaf(y[i], 0.f, odd);
    if (std::is_same<T, __nv_bfloat16>::value && odd == 0.f) {
#pragma unroll
        for (int i = 0; i < N; i += 2)
            w[i / 2] = __byte_perm(__float_as_uint(y[i]) + (random[i] * 0x9e3779b1u >> 16), __float_as_uint(y[i + 1]) + (random[i + 1] * 0x9e3779b1u >> 16), 0x7632);
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) w[i / 2] = round_random<T>(y[i], random[i] * 0x9e3779b1u) | round_random<T>(y[i + 1], random[i + 1] * 0x9e3779b1u) << 16;
    }
#pragma unroll
    for (int j = 0; j < N / 8; ++j) raw[j] = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
}

__device__ double power(double b, int64_t t)
{
    double r = 1.0;
    for (; t > 0; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

__device__ __forceinline__ float root_of(float x)
{
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float root_flushed(float x)
{
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// a / b; b is 0 or a normal number far from the largest, and quotients below 2^-126 change no weight
__device__ __forceinline__ float quotient(float a, float b)
{
    float y;
    asm("div.approx.ftz.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

template <class P, class G, int BITS, bool MASTER, bool RANDOM, int CAP>
__global__ void __launch_bounds__(kThreads<BITS>) step_kernel(const __grid_constant__ Table<CAP> table, const __grid_constant__ StepArgs s)
{
    if (s.skip && *s.skip != 0.f) return;
    __shared__ float derived[3];
    float rate = s.rate, root = s.root;
    double lr = s.lr;
    uint32_t key = s.key;
    if (s.step_device || s.lr_device) {  // a captured step reads its number and rate when it is replayed
        const int64_t t = max(s.step_device ? *s.step_device : 1ll, 1ll);
        if (s.lr_device) lr = *s.lr_device;
        if (threadIdx.x == 0) derived[0] = static_cast<float>(lr / (1.0 - power(s.beta1, t)));
        if (threadIdx.x == 32) derived[1] = static_cast<float>(1.0 / sqrt(1.0 - power(s.beta2, t)));
        __syncthreads();
        if (s.step_device) key = mix(mix(s.seed) + static_cast<uint32_t>(t));
        rate = derived[0], root = derived[1];
    }
    const float scale = s.grad_scale ? *s.grad_scale : 1.f;
    uint32_t at = tensor_of(table, blockIdx.x);
    for (uint32_t chunk = blockIdx.x; chunk < table.chunks; chunk += gridDim.x) {
        while (at + 1 < table.count && chunk >= table.e[at + 1].first) ++at;
        const Entry &t = table.e[at];
        constexpr int N = kPer<BITS>;
        using W = typename std::conditional<MASTER, float, P>::type;  // what is stepped
        using M = typename std::conditional<BITS == 32, float, uint8_t>::type;
        constexpr int kW = N * static_cast<int>(sizeof(W)) / 16, kG = N * static_cast<int>(sizeof(G)) / 16, kM = N * static_cast<int>(sizeof(M)) / 16;
        const int64_t e = static_cast<int64_t>(chunk - t.first) * kChunk + threadIdx.x * N;
        const int left = static_cast<int>(min(t.n - e, static_cast<int64_t>(N)));  // not above 0 behind the tensor's end
        const bool all = left == N, whole = all && (t.flags & kWide);
        W *weights = MASTER ? reinterpret_cast<W *>(t.master) : static_cast<W *>(t.param);
        uint4 rw[kW], rg[kG], rm[kM], rv[kM];
        load<W, N>(weights + e, left, whole, rw);
        load<G, N>(static_cast<const G *>(t.grad) + e, left, whole, rg);
        const bool states = all && (BITS == 8 || (t.flags & kWideStates));
        load<M, N>(static_cast<const M *>(t.m) + e, left, states, rm);
        load<M, N>(static_cast<const M *>(t.v) + e, left, states, rv);
        float p[N], m[N], v[N];
        if constexpr (BITS == 32) {
            unpack<float, N>(rm, m), unpack<float, N>(rv, v);
        } else {
            const uint32_t em = left > 0 ? t.m_exp[e / kBlock] : 0, ev = left > 0 ? t.v_exp[e / kBlock] : 0;
            decode<true, N>(reinterpret_cast<const uint32_t *>(rm), em, m), decode<false, N>(reinterpret_cast<const uint32_t *>(rv), ev, v);
            if (!all)  // a block that is not finite has nothing behind the tensor's end
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (i >= left) m[i] = v[i] = 0.f;
        }
        const float decay = s.lr_device ? static_cast<float>(1.0 - lr * static_cast<double>(t.weight_decay)) : t.decay;
        const bool keep = t.flags & kKeepZeros;
        float g[N];
        unpack<W, N>(rw, p), unpack<G, N>(rg, g);
        if (s.grad_scale)
#pragma unroll
            for (int i = 0; i < N; ++i) g[i] *= scale;
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            // Two elements an instruction (100 M of them in 8 bits 221 -> 210 us, bound by instructions), every product and sum
            // rounded by itself: the 8-bit codes below are those of the plain formula, bit for bit.
            float2 first = make_float2(m[i], m[i + 1]), second = make_float2(v[i], v[i + 1]);
            const float2 slope = make_float2(g[i], g[i + 1]);
            first = __fadd2_rn(__fmul2_rn(first, both(s.b1)), __fmul2_rn(slope, both(s.g1)));
            second = __fadd2_rn(__fmul2_rn(second, both(s.b2)), __fmul2_rn(__fmul2_rn(slope, both(s.g2)), slope));
            m[i] = first.x, m[i + 1] = first.y, v[i] = second.x, v[i + 1] = second.y;
        }
        if (keep)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (p[i] == 0.f) m[i] = v[i] = 0.f;
        // Roots of numbers below 2^-126, 2^-63 times `root`, do not show beside such an eps; and with finite rate and decay a weight of 0 whose m is
        // 0 stays 0 by itself.
        if (s.eps >= 1e-9f && s.eps >= 1e-12f * root && fabsf(rate) <= 3.4e38f && fabsf(decay) <= 3.4e38f) {
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const float2 above = __fmul2_rn(make_float2(m[i], m[i + 1]), both(rate)), below = __ffma2_rn(make_float2(root_flushed(v[i]), root_flushed(v[i + 1])), both(root), both(s.eps));
                const float2 next = __ffma2_rn(make_float2(p[i], p[i + 1]), both(decay), make_float2(-quotient(above.x, below.x), -quotient(above.y, below.y)));
                p[i] = next.x, p[i + 1] = next.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float below = fmaf(root_of(v[i]), root, s.eps), up = below < 0x1p-60f ? 0x1p60f : 1.f;  // numbers below 2^-126 would count as 0
                p[i] = keep && p[i] == 0.f ? 0.f : fmaf(p[i], decay, -quotient(m[i] * rate * up, below * up));
            }
        }
        uint32_t random[N];
        if (BITS == 8 || RANDOM) {
            const uint32_t start = mix(key + t.index) + static_cast<uint32_t>(e) + static_cast<uint32_t>(e >> 32) * 0x9e3779b9u;
#pragma unroll
            for (int i = 0; i < N; ++i) random[i] = mix(start + i);
        }
        if (MASTER) store<W, N>(weights + e, left, whole, (pack<W, N>(p, rw), rw));
        uint4 rp[N * static_cast<int>(sizeof(P)) / 16];
        if constexpr (RANDOM) pack_random<P, N>(p, random, rp);
        else pack<P, N>(p, rp);
        store<P, N>(static_cast<P *>(t.param) + e, left, whole, rp);
        if constexpr (BITS == 32) {
            pack<float, N>(m, rm), pack<float, N>(v, rv);
        } else {
            uint32_t em, ev;
            encode<true, N>(m, random, reinterpret_cast<uint32_t *>(rm), em), encode<false, N>(v, random, reinterpret_cast<uint32_t *>(rv), ev);
            if (left > 0 && threadIdx.x % (kBlock / N) == 0) t.m_exp[e / kBlock] = static_cast<uint8_t>(em), t.v_exp[e / kBlock] = static_cast<uint8_t>(ev);
        }
        store<M, N>(static_cast<M *>(t.m) + e, left, states, rm);
        store<M, N>(static_cast<M *>(t.v) + e, left, states, rv);
    }
}

// Moments in 8 bits as numbers.  param and master of the table: where the first and the second go.
template <class T, int CAP> __global__ void __launch_bounds__(kThreads<8>) moments_kernel(const __grid_constant__ Table<CAP> table)
{
    constexpr int N = kPer<8>;
    uint32_t at = tensor_of(table, blockIdx.x);
    for (uint32_t chunk = blockIdx.x; chunk < table.chunks; chunk += gridDim.x) {
        while (at + 1 < table.count && chunk >= table.e[at + 1].first) ++at;
        const Entry &t = table.e[at];
        const int64_t e = static_cast<int64_t>(chunk - t.first) * kChunk + threadIdx.x * N;
        const int left = static_cast<int>(min(t.n - e, static_cast<int64_t>(N)));
        if (left <= 0) continue;
        const bool all = left == N, whole = all && (t.flags & kWide);
        uint4 rm, rv, out[N * static_cast<int>(sizeof(T)) / 16];
        load<uint8_t, N>(static_cast<const uint8_t *>(t.m) + e, left, all, &rm), load<uint8_t, N>(static_cast<const uint8_t *>(t.v) + e, left, all, &rv);
        float y[N];
        decode<true, N>(reinterpret_cast<const uint32_t *>(&rm), t.m_exp[e / kBlock], y);
        pack<T, N>(y, out);
        store<T, N>(static_cast<T *>(t.param) + e, left, whole, out);
        decode<false, N>(reinterpret_cast<const uint32_t *>(&rv), t.v_exp[e / kBlock], y);
        pack<T, N>(y, out);
        store<T, N>(reinterpret_cast<T *>(t.master) + e, left, whole, out);
    }
}

// ---------------------------------------------------------------------------------------------- launches
// A block per chunk: with blocks that walk over several, fp32 states ran at 5.5 TB/s instead of 6.4 (a block's loads wait for its stores).
// Where each block has to work out the step's numbers first, only as many as can be resident.
template <class K, int CAP, class... A> int launch(K kernel, int threads, bool resident, const Table<CAP> &table, cudaStream_t stream, A... more)
{
    const uint32_t most = resident ? static_cast<uint32_t>(sm_count()) * (2048 / threads) : 0x7fffffffu;
    kernel<<<table.chunks < most ? table.chunks : most, threads, 0, stream>>>(table, more...);
    return finish_launch();
}

// Calls `go` with the tensors that `wanted` names, as many at a time as a launch takes.
template <int CAP, class Wanted, class Fill, class Go> int batches(int32_t count, const spdy_adamw_tensor *tensors, Wanted wanted, Fill fill, Go go)
{
    Table<CAP> table;
    table.count = table.chunks = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (!wanted(tensors[i])) continue;
        const int64_t chunks = (tensors[i].n + kChunk - 1) / kChunk;
        if (table.count == CAP || (table.count && chunks + table.chunks > 0x7fffffff)) {
            const int rc = go(table);
            if (rc != SPDY_OK) return rc;
            table.count = table.chunks = 0;
        }
        Entry &e = table.e[table.count++];
        fill(e, i);
        e.first = table.chunks, e.n = tensors[i].n, e.index = static_cast<uint32_t>(i);
        table.chunks += static_cast<uint32_t>(chunks);
    }
    return table.count ? go(table) : SPDY_OK;
}
template <class Wanted, class Fill, class GoFew, class GoMany>
int all_batches(int32_t count, const spdy_adamw_tensor *tensors, Wanted wanted, Fill fill, GoFew few, GoMany many)
{
    int n = 0;
    for (int32_t i = 0; i < count; ++i) n += wanted(tensors[i]) ? 1 : 0;
    if (n == 0) return SPDY_OK;
    return n <= kFew ? batches<kFew>(count, tensors, wanted, fill, few) : batches<kMany>(count, tensors, wanted, fill, many);
}

template <class P, class G, int BITS, bool MASTER, bool RANDOM> int step_kind(int32_t count, const spdy_adamw_tensor *tensors, int ptype, int gtype, const StepArgs &s, cudaStream_t stream)
{
    const auto wanted = [&](const spdy_adamw_tensor &t) {
        return t.grad && t.n > 0 && t.param_dtype == ptype && t.grad_dtype == gtype && t.state_bits == BITS && (t.master != nullptr) == MASTER;
    };
    const auto fill = [&](Entry &e, int32_t i) {
        const spdy_adamw_tensor &t = tensors[i];
        e.param = t.param, e.grad = t.grad, e.master = t.master, e.m = t.m, e.v = t.v, e.m_exp = t.m_exp, e.v_exp = t.v_exp;
        e.weight_decay = t.weight_decay, e.decay = static_cast<float>(1.0 - s.lr * static_cast<double>(t.weight_decay));
        e.flags = (aligned(t.param, 32) && aligned(t.grad, 32) && aligned(t.master, 32) ? kWide : 0) | (aligned(t.m, 32) && aligned(t.v, 32) ? kWideStates : 0) | (t.keep_zeros ? kKeepZeros : 0);
    };
    const auto go = [&](const auto &table) {
        constexpr int cap = static_cast<int>(sizeof(table.e) / sizeof(Entry));
        return launch(step_kernel<P, G, BITS, MASTER, RANDOM, cap>, kThreads<BITS>, s.step_device != nullptr, table, stream, s);
    };
    return all_batches(count, tensors, wanted, fill, go, go);
}

template <class P, class G, int BITS> int step_copies(int32_t count, const spdy_adamw_tensor *tensors, int ptype, int gtype, bool random, const StepArgs &s, cudaStream_t stream)
{
    if constexpr (sizeof(P) == 2) {
        const int rc = step_kind<P, G, BITS, true, false>(count, tensors, ptype, gtype, s, stream);
        if (rc != SPDY_OK) return rc;
        if (random) return step_kind<P, G, BITS, false, true>(count, tensors, ptype, gtype, s, stream);
    }
    return step_kind<P, G, BITS, false, false>(count, tensors, ptype, gtype, s, stream);
}
template <class P, class G> int step_types(int32_t count, const spdy_adamw_tensor *tensors, int ptype, int gtype, bool random, const StepArgs &s, cudaStream_t stream)
{
    const int rc = step_copies<P, G, 32>(count, tensors, ptype, gtype, random, s, stream);
    return rc != SPDY_OK ? rc : step_copies<P, G, 8>(count, tensors, ptype, gtype, random, s, stream);
}

bool states_ok(const spdy_adamw_tensor &t)
{
    if (t.state_bits != 32 && t.state_bits != 8) return false;
    if (t.n == 0) return true;
    return t.m && t.v && aligned(t.m, 16) && aligned(t.v, 16) && (t.state_bits == 32 || (t.m_exp && t.v_exp));
}
constexpr int64_t kMostElements = 1ll << 41;  // chunks of one tensor are counted in 32 bits

bool tensor_ok(const spdy_adamw_tensor &t)
{
    if (t.n < 0 || t.n > kMostElements || !known_type(t.param_dtype) || !states_ok(t) || !(t.weight_decay >= 0.f && t.weight_decay <= 3.4e38f)) return false;
    if (t.grad && t.grad_dtype != t.param_dtype && t.grad_dtype != SPDY_F32) return false;
    if (t.master && t.param_dtype == SPDY_F32) return false;
    return t.n == 0 || (t.param && aligned(t.param, type_size(t.param_dtype)) && aligned(t.master, 4) && (!t.grad || aligned(t.grad, type_size(t.grad_dtype))));
}

}  // namespace

extern "C" {

int spdy_adamw_step(const spdy_adamw_tensor *tensors, int32_t count, const spdy_adamw_options *o, void *cuda_stream)
{
    if (count < 0 || (count > 0 && !tensors) || !o) return SPDY_ERR_INVALID_ARG;
    const auto part = [](double b) { return b >= 0.0 && b < 1.0; };
    if (!part(o->beta1) || !part(o->beta2) || !(o->eps >= 0.0 && o->eps <= 1e30) || (o->rounding != 0 && o->rounding != 1)) return SPDY_ERR_INVALID_ARG;
    if ((!o->lr_device && !(o->lr >= 0.0 && o->lr <= 1e30)) || (!o->step_device && o->step < 1)) return SPDY_ERR_INVALID_ARG;
    if (!aligned(o->lr_device, 4) || !aligned(o->step_device, 8) || !aligned(o->grad_scale, 4) || !aligned(o->skip, 4)) return SPDY_ERR_INVALID_ARG;
    for (int32_t i = 0; i < count; ++i)
        if (!tensor_ok(tensors[i])) return SPDY_ERR_INVALID_ARG;
    StepArgs s = {};
    s.b1 = static_cast<float>(o->beta1), s.b2 = static_cast<float>(o->beta2);
    s.g1 = static_cast<float>(1.0 - o->beta1), s.g2 = static_cast<float>(1.0 - o->beta2);
    s.eps = o->eps > 0.0 ? fmaxf(static_cast<float>(o->eps), 0x1p-149f) : 0.f;  // one that is there does not become 0: 0 / eps is 0
    s.lr = o->lr, s.beta1 = o->beta1, s.beta2 = o->beta2;
    const double t = static_cast<double>(o->step);
    s.rate = static_cast<float>(o->lr / (1.0 - pow(o->beta1, t))), s.root = static_cast<float>(1.0 / sqrt(1.0 - pow(o->beta2, t)));
    s.seed = o->seed, s.key = mix(mix(o->seed) + static_cast<uint32_t>(o->step));
    s.lr_device = o->lr_device, s.step_device = o->step_device, s.grad_scale = o->grad_scale, s.skip = o->skip;
    if (s.lr_device && !s.step_device) return SPDY_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool random = o->rounding == 1;
    int rc = step_types<float, float>(count, tensors, SPDY_F32, SPDY_F32, random, s, stream);
    if (rc == SPDY_OK) rc = step_types<__nv_bfloat16, __nv_bfloat16>(count, tensors, SPDY_BF16, SPDY_BF16, random, s, stream);
    if (rc == SPDY_OK) rc = step_types<__nv_bfloat16, float>(count, tensors, SPDY_BF16, SPDY_F32, random, s, stream);
    if (rc == SPDY_OK) rc = step_types<__half, __half>(count, tensors, SPDY_F16, SPDY_F16, random, s, stream);
    if (rc == SPDY_OK) rc = step_types<__half, float>(count, tensors, SPDY_F16, SPDY_F32, random, s, stream);
    return rc;
}

int spdy_adamw_moments(const spdy_adamw_tensor *tensors, int32_t count, void *const *m_out, void *const *v_out, int out_dtype, void *cuda_stream)
{
    if (count < 0 || (count > 0 && (!tensors || !m_out || !v_out)) || (out_dtype != SPDY_F32 && out_dtype != SPDY_BF16)) return SPDY_ERR_INVALID_ARG;
    for (int32_t i = 0; i < count; ++i) {
        if (tensors[i].n < 0 || tensors[i].n > kMostElements || !states_ok(tensors[i]) || tensors[i].state_bits != 8) return SPDY_ERR_INVALID_ARG;
        if (tensors[i].n > 0 && (!m_out[i] || !v_out[i] || !aligned(m_out[i], type_size(out_dtype)) || !aligned(v_out[i], type_size(out_dtype)))) return SPDY_ERR_INVALID_ARG;
    }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const auto wanted = [](const spdy_adamw_tensor &t) { return t.n > 0; };
    const auto fill = [&](Entry &e, int32_t i) {
        const spdy_adamw_tensor &t = tensors[i];
        e = {};
        e.param = m_out[i], e.master = static_cast<float *>(v_out[i]), e.m = t.m, e.v = t.v, e.m_exp = t.m_exp, e.v_exp = t.v_exp;
        e.flags = aligned(m_out[i], 32) && aligned(v_out[i], 32) ? kWide : 0;
    };
    const auto go = [&](const auto &table) {
        constexpr int cap = static_cast<int>(sizeof(table.e) / sizeof(Entry));
        return out_dtype == SPDY_F32 ? launch(moments_kernel<float, cap>, kThreads<8>, false, table, stream) : launch(moments_kernel<__nv_bfloat16, cap>, kThreads<8>, false, table, stream);
    };
    return all_batches(count, tensors, wanted, fill, go, go);
}

}  // extern "C"
