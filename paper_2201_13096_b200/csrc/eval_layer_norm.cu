// Layer normalisation and its gradients: kernels and C entries (spdy_eval.h).
//
// Both directions read every element once and keep a row's part in registers between the two sums it needs (the mean before
// the squared deviations; sum u and sum u h before dx), so they are bound by memory.  A row belongs to one warp while it
// fits (no barrier then; short rows share a warp), to 128 to 1024 threads when it is longer, and beyond that it is read again per sum.
#include "eval_common.cuh"

using namespace spdy_eval;

namespace {

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    int64_t ldx, lddy, ldy, lddx, R, D;
    int param_type;
    int params_wide;                // bit 0: weight starts on 16 bytes, bit 1: bias
    float eps;
    void *y, *dx;
    float *mean, *rstd;             // forward's results
    const float *in_mean, *in_rstd; // backward's inputs
    float *partial;                 // [blocks][2][D]
    int want_params;                // dweight or dbias asked for
};

// The type of weight and bias as the kernels see it: T's own or fp32 (the choice is a template argument of the hot kernels).
__device__ __forceinline__ float param_at(const void *p, int type, int64_t i)
{
    if (type == SPDY_F32) return static_cast<const float *>(p)[i];
    if (type == SPDY_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(static_cast<const __half *>(p)[i]);
}

// N values from index e on, `fallback` for a NULL vector and outside [0, D).  `wide`: p starts on 16 bytes.
template <class P, int N> __device__ __forceinline__ void params(const void *p, bool wide, int e, int D, float fallback, float *f)
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = fallback;
        return;
    }
    const P *at = static_cast<const P *>(p) + e;
    constexpr int PV = Elem<P>::kVec;
    if (N % PV == 0 && wide && e % PV == 0 && e + N <= D) {
#pragma unroll
        for (int i = 0; i + PV <= N; i += PV) Elem<P>::unpack(*reinterpret_cast<const uint4 *>(at + i), f + i);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = e + i >= 0 && e + i < D ? Elem<P>::to_float(at[i]) : fallback;
}

// Sums of TPR consecutive threads' values, in all of them.  `slot` alternates between calls, so that one barrier is enough.
template <int TPR, int COUNT> __device__ __forceinline__ void row_sums(float *v, float (*shared)[32], int slot)
{
#pragma unroll
    for (int d = TPR < 32 ? TPR / 2 : 16; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    if (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) shared[slot * COUNT + i][warp] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            v[i] = lane < W ? shared[slot * COUNT + i][lane] : 0.f;
#pragma unroll
            for (int d = 16; d; d >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
        }
    }
}

// A group of TPR threads holds a row in registers: granule v * TPR + t belongs to its thread t.  WHOLE: every granule of every row
// lies wholly inside it (aligned rows of a multiple of 16 bytes), so that no element needs a test.
template <class T, class P, int TPR, int VPT, int NT, bool WHOLE> __global__ void __launch_bounds__(NT) norm_forward_kernel(const NormArgs a)
{
    constexpr int VEC = Elem<T>::kVec;
    __shared__ float shared[2][32];
    const int64_t r = static_cast<int64_t>(blockIdx.x) * (NT / TPR) + threadIdx.x / TPR;
    const bool here = r < a.R;  // the last block's spare groups take part in the warp's sums
    const int t = threadIdx.x % TPR;
    const Row<T> row(static_cast<const T *>(a.x) + (here ? r : 0) * a.ldx, a.D);
    const int G = here ? row.granules() : 0;
    uint4 raw[VPT];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int g = v * TPR + t;
        if (g < G) raw[v] = WHOLE ? load_stream(row.p + g * VEC) : row.load(g);
    }
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int g = v * TPR + t;
        if (g >= G) continue;
        float f[VEC];
        Elem<T>::unpack(raw[v], f);
        const int e = row.first(g);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (WHOLE || (e + i >= 0 && e + i < row.n)) sum += f[i];
    }
    row_sums<TPR, 1>(&sum, shared, 0);
    const float n = static_cast<float>(a.D), mean = sum / n;
    float sq = 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int g = v * TPR + t;
        if (g >= G) continue;
        float f[VEC];
        Elem<T>::unpack(raw[v], f);
        const int e = row.first(g);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (WHOLE || (e + i >= 0 && e + i < row.n)) sq = fmaf(f[i] - mean, f[i] - mean, sq);
    }
    row_sums<TPR, 1>(&sq, shared, 1);
    const float rstd = 1.f / sqrtf(sq / n + a.eps);
    if (t == 0 && here) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    T *out = static_cast<T *>(a.y) + r * a.ldy;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int g = v * TPR + t;
        if (g >= G) continue;
        const int e = WHOLE ? g * VEC : row.first(g);
        float f[VEC], w[VEC], b[VEC];
        Elem<T>::unpack(raw[v], f);
        params<P, VEC>(a.weight, a.params_wide & 1, e, row.n, 1.f, w);
        params<P, VEC>(a.bias, a.params_wide & 2, e, row.n, 0.f, b);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = fmaf((f[i] - mean) * rstd, w[i], b[i]);
        const uint4 packed = Elem<T>::pack(f);
        if (WHOLE || (row.same_lead(out) && row.whole(g))) store_stream(out + e, packed);
        else store_part(out, row.n, e, packed);
    }
}

// Rows too long for the registers of a block: one block per row, the row read once per sum (from L2 after the first).
template <class T, int NT> __global__ void __launch_bounds__(NT) norm_forward_long_kernel(const NormArgs a)
{
    __shared__ float shared[2][32];
    const int64_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + r * a.ldx;
    T *out = static_cast<T *>(a.y) + r * a.ldy;
    float sum = 0.f, sq = 0.f;
    for (int64_t i = threadIdx.x; i < a.D; i += NT) sum += Elem<T>::to_float(x[i]);
    row_sums<NT, 1>(&sum, shared, 0);
    const float n = static_cast<float>(a.D), mean = sum / n;
    for (int64_t i = threadIdx.x; i < a.D; i += NT) {
        const float d = Elem<T>::to_float(x[i]) - mean;
        sq = fmaf(d, d, sq);
    }
    row_sums<NT, 1>(&sq, shared, 1);
    const float rstd = 1.f / sqrtf(sq / n + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    for (int64_t i = threadIdx.x; i < a.D; i += NT) {
        const float w = a.weight ? param_at(a.weight, a.param_type, i) : 1.f, b = a.bias ? param_at(a.bias, a.param_type, i) : 0.f;
        out[i] = Elem<T>::from_float(fmaf((Elem<T>::to_float(x[i]) - mean) * rstd, w, b));
    }
}

// What a thread of the backward kernel holds of a row: VPT times 16 bytes (WIDE: rows start on 16 bytes; the last ones may be
// partly outside and read as 0 there), or VPT single elements.
template <class T, int VPT, bool WIDE> struct Held;
template <class T, int VPT> struct Held<T, VPT, true> {
    static constexpr int kVec = Elem<T>::kVec;
    uint4 raw[VPT];
    __device__ __forceinline__ void load(const T *p, int n, int t, int threads)
    {
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = (v * threads + t) * kVec;
            raw[v] = make_uint4(0, 0, 0, 0);
            if (e + kVec <= n) {
                raw[v] = load_stream(p + e);
            } else if (e < n) {
                float f[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) f[i] = e + i < n ? Elem<T>::to_float(p[e + i]) : 0.f;
                raw[v] = Elem<T>::pack(f);
            }
        }
    }
    __device__ __forceinline__ void get(int v, float *f) const { Elem<T>::unpack(raw[v], f); }
    // what was unpacked is unpacked again rather than kept in twice the registers
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int v = 0; v < VPT; ++v) asm volatile("" : "+r"(raw[v].x), "+r"(raw[v].y), "+r"(raw[v].z), "+r"(raw[v].w));
    }
    static __device__ __forceinline__ void store(T *p, int n, int e, const float *f)
    {
        if (e + kVec <= n && (reinterpret_cast<uintptr_t>(p + e) & 15) == 0) store_stream(p + e, Elem<T>::pack(f));
        else store_part(p, n, e, Elem<T>::pack(f));
    }
};
template <class T, int VPT> struct Held<T, VPT, false> {
    static constexpr int kVec = 1;
    T raw[VPT];
    __device__ __forceinline__ void load(const T *p, int n, int t, int threads)
    {
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = v * threads + t;
            raw[v] = e < n ? p[e] : Elem<T>::from_float(0.f);
        }
    }
    __device__ __forceinline__ void get(int v, float *f) const { f[0] = Elem<T>::to_float(raw[v]); }
    __device__ __forceinline__ void forget() {}
    static __device__ __forceinline__ void store(T *p, int, int e, const float *f) { p[e] = Elem<T>::from_float(f[0]); }
};

// Each group of TPR threads walks over rows, the next row's elements on their way while this one's are used, and keeps the sums of
// its columns for dweight and dbias in registers; the groups of a block are joined through shared memory in a fixed order,
// the blocks by norm_columns_kernel.
template <class T, class P, int TPR, int VPT, bool WIDE, bool AHEAD, int NT> __global__ void __launch_bounds__(NT) norm_backward_kernel(const NormArgs a)
{
    constexpr int GROUPS = NT / TPR, VEC = Held<T, VPT, WIDE>::kVec;
    __shared__ float shared[4][32];
    extern __shared__ float columns[];  // [GROUPS - 1][2][D]
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, D = static_cast<int>(a.D);
    float dw[VPT * VEC], db[VPT * VEC];
#pragma unroll
    for (int i = 0; i < VPT * VEC; ++i) dw[i] = db[i] = 0.f;
    const float inv_n = 1.f / static_cast<float>(a.D);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * GROUPS;
    Held<T, VPT, WIDE> x, dy, next_x, next_dy;
    float mean = 0.f, rstd = 0.f, next_mean = 0.f, next_rstd = 0.f;
    const auto fetch = [&](int64_t r, Held<T, VPT, WIDE> &to_x, Held<T, VPT, WIDE> &to_dy, float &to_mean, float &to_rstd) {
        const int n = r < a.R ? D : 0;  // a spare group's row: nothing is read, everything is 0
        const int64_t at = r < a.R ? r : 0;
        to_x.load(static_cast<const T *>(a.x) + at * a.ldx, n, t, TPR);
        to_dy.load(static_cast<const T *>(a.dy) + at * a.lddy, n, t, TPR);
        to_mean = a.in_mean[at], to_rstd = a.in_rstd[at];
    };
    if (AHEAD) fetch(static_cast<int64_t>(blockIdx.x) * GROUPS + group, next_x, next_dy, next_mean, next_rstd);
    int slot = 0;
    // the same number of rounds for all groups of a block: their threads meet in the sums
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * GROUPS; base < a.R; base += stride, slot ^= 1) {
        const int64_t r = base + group;
        const bool here = r < a.R;
        if (AHEAD) {
            x = next_x, dy = next_dy, mean = next_mean, rstd = next_rstd;
            if (base + stride < a.R) fetch(r + stride, next_x, next_dy, next_mean, next_rstd);
        } else {
            fetch(r, x, dy, mean, rstd);
        }
        T *out = static_cast<T *>(a.dx) + r * a.lddx;
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = (v * TPR + t) * VEC;
            if (e >= D || !here) continue;
            float w[VEC], h[VEC], u[VEC];
            params<P, VEC>(a.weight, a.params_wide & 1, e, D, 1.f, w);
            x.get(v, h), dy.get(v, u);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int k = v * VEC + i;
                const float hat = (h[i] - mean) * rstd;  // beyond the row dy is 0, and so is all that follows
                dw[k] = fmaf(u[i], hat, dw[k]);
                db[k] += u[i];
                u[i] *= w[i];
                sums[0] += u[i];
                sums[1] = fmaf(u[i], hat, sums[1]);
            }
        }
        row_sums<TPR, 2>(sums, shared, slot);
        const float mu = sums[0] * inv_n, mh = sums[1] * inv_n;
        x.forget(), dy.forget();
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = (v * TPR + t) * VEC;
            if (e >= D || !here) continue;
            float w[VEC], h[VEC], f[VEC];
            params<P, VEC>(a.weight, a.params_wide & 1, e, D, 1.f, w);
            x.get(v, h), dy.get(v, f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = rstd * (f[i] * w[i] - fmaf((h[i] - mean) * rstd, mh, mu));
            Held<T, VPT, WIDE>::store(out, D, e, f);
        }
    }
    if (!a.want_params) return;
    if (GROUPS > 1) {
        if (group > 0) {
#pragma unroll
            for (int k = 0; k < VPT * VEC; ++k) {
                const int e = ((k / VEC) * TPR + t) * VEC + k % VEC;
                if (e < D) columns[(group - 1) * 2 * D + e] = dw[k], columns[(group - 1) * 2 * D + D + e] = db[k];
            }
        }
        __syncthreads();
        if (group > 0) return;
        for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
            for (int k = 0; k < VPT * VEC; ++k) {
                const int e = ((k / VEC) * TPR + t) * VEC + k % VEC;
                if (e < D) dw[k] += columns[g * 2 * D + e], db[k] += columns[g * 2 * D + D + e];
            }
    }
    float *to = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * D;
#pragma unroll
    for (int k = 0; k < VPT * VEC; ++k) {
        const int e = ((k / VEC) * TPR + t) * VEC + k % VEC;
        if (e < D) to[e] = dw[k], to[D + e] = db[k];
    }
}

// Long rows: dx with one block per row, the columns' sums by a second kernel over blocks of columns and rows.
template <class T, int NT> __global__ void __launch_bounds__(NT) norm_backward_long_kernel(const NormArgs a)
{
    __shared__ float shared[2][32];
    const int64_t r = blockIdx.x;
    const T *x = static_cast<const T *>(a.x) + r * a.ldx, *dy = static_cast<const T *>(a.dy) + r * a.lddy;
    T *out = static_cast<T *>(a.dx) + r * a.lddx;
    const float mean = a.in_mean[r], rstd = a.in_rstd[r];
    float sums[2] = {0.f, 0.f};
    for (int64_t i = threadIdx.x; i < a.D; i += NT) {
        const float u = Elem<T>::to_float(dy[i]) * (a.weight ? param_at(a.weight, a.param_type, i) : 1.f);
        sums[0] += u;
        sums[1] = fmaf(u, (Elem<T>::to_float(x[i]) - mean) * rstd, sums[1]);
    }
    row_sums<NT, 2>(sums, shared, 0);
    const float inv_n = 1.f / static_cast<float>(a.D), mu = sums[0] * inv_n, mh = sums[1] * inv_n;
    for (int64_t i = threadIdx.x; i < a.D; i += NT) {
        const float u = Elem<T>::to_float(dy[i]) * (a.weight ? param_at(a.weight, a.param_type, i) : 1.f);
        out[i] = Elem<T>::from_float(rstd * (u - fmaf((Elem<T>::to_float(x[i]) - mean) * rstd, mh, mu)));
    }
}

template <class T> __global__ void __launch_bounds__(256) norm_backward_columns_kernel(const NormArgs a, int64_t rows_per_block)
{
    const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (e >= a.D) return;
    const int64_t r0 = blockIdx.y * rows_per_block, r1 = min(a.R, r0 + rows_per_block);
    float dw = 0.f, db = 0.f;
    for (int64_t r = r0; r < r1; ++r) {
        const float g = Elem<T>::to_float(static_cast<const T *>(a.dy)[r * a.lddy + e]);
        dw = fmaf(g, (Elem<T>::to_float(static_cast<const T *>(a.x)[r * a.ldx + e]) - a.in_mean[r]) * a.in_rstd[r], dw);
        db += g;
    }
    a.partial[blockIdx.y * 2 * a.D + e] = dw;
    a.partial[blockIdx.y * 2 * a.D + a.D + e] = db;
}

// dweight and dbias from the blocks' sums, 32 columns per block, each of 32 warps adding every 32nd block's.
__global__ void __launch_bounds__(1024) norm_columns_kernel(const float *partial, int blocks, int64_t D, float *dweight, float *dbias)
{
    __shared__ float part[32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t e = static_cast<int64_t>(blockIdx.x) * 32 + lane;  // over [2][D], each half rounded up to 32
    const int64_t padded = (D + 31) / 32 * 32;
    const bool second = static_cast<int64_t>(blockIdx.x) * 32 >= padded;
    const int64_t col = second ? e - padded : e;
    float sum = 0.f;
    if (col < D) {
        const float *p = partial + (second ? D : 0) + col;
#pragma unroll 8
        for (int b = warp; b < blocks; b += 32) sum += p[static_cast<int64_t>(b) * 2 * D];
    }
    part[warp][lane] = sum;
    __syncthreads();
    // warp w takes column w: its 32 sums in a tree
    sum = part[lane][warp];
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const int64_t mine = (second ? static_cast<int64_t>(blockIdx.x) * 32 - padded : static_cast<int64_t>(blockIdx.x) * 32) + warp;
    float *to = second ? dbias : dweight;
    if (lane == 0 && to && mine < D) to[mine] = sum;
}

template <class T, int TPR, int VPT, int NT> int forward_with(const NormArgs &a, bool whole, cudaStream_t s)
{
    const unsigned blocks = static_cast<unsigned>((a.R + NT / TPR - 1) / (NT / TPR));
    if (a.param_type == SPDY_F32) {
        if (whole) norm_forward_kernel<T, float, TPR, VPT, NT, true><<<blocks, NT, 0, s>>>(a);
        else norm_forward_kernel<T, float, TPR, VPT, NT, false><<<blocks, NT, 0, s>>>(a);
    } else {
        if (whole) norm_forward_kernel<T, T, TPR, VPT, NT, true><<<blocks, NT, 0, s>>>(a);
        else norm_forward_kernel<T, T, TPR, VPT, NT, false><<<blocks, NT, 0, s>>>(a);
    }
    return finish_launch();
}

template <class T> int forward(const NormArgs &a, cudaStream_t s)
{
    constexpr int VEC = Elem<T>::kVec;
    if (a.R > 0x7fffffff) return SPDY_ERR_UNSUPPORTED;
    const bool in_line = a.ldx % VEC == 0 && aligned(a.x, 16);
    const bool whole = in_line && a.ldy % VEC == 0 && aligned(a.y, 16) && a.D % VEC == 0;
    const int64_t G = (a.D + VEC - 1) / VEC + (in_line ? 0 : 1);
    // Short rows share a warp; a row stays with one warp (no barrier) up to 8 granules a thread.
    if (G <= 4) return forward_with<T, 4, 1, 128>(a, whole, s);
    if (G <= 8) return forward_with<T, 8, 1, 128>(a, whole, s);
    if (G <= 16) return forward_with<T, 16, 1, 128>(a, whole, s);
    if (G <= 32) return forward_with<T, 32, 1, 128>(a, whole, s);
    if (G <= 64) return forward_with<T, 32, 2, 128>(a, whole, s);
    if (G <= 96) return forward_with<T, 32, 3, 128>(a, whole, s);
    if (G <= 128) return forward_with<T, 32, 4, 128>(a, whole, s);
    if (G <= 256) return forward_with<T, 32, 8, 128>(a, whole, s);
    if (G <= 512) return forward_with<T, 128, 4, 128>(a, whole, s);
    if (G <= 1024) return forward_with<T, 256, 4, 256>(a, whole, s);
    if (G <= 2048) return forward_with<T, 512, 4, 512>(a, whole, s);
    if (G <= 4096) return forward_with<T, 1024, 4, 1024>(a, whole, s);
    norm_forward_long_kernel<T, 512><<<static_cast<unsigned>(a.R), 512, 0, s>>>(a);
    return finish_launch();
}

// How the backward kernel holds rows of D columns: threads per row, columns per thread.  Wide rows: up to 32 columns a thread
// (64 sums in registers), single elements: up to 16.
struct BackwardShape {
    int threads, columns, block;
};
BackwardShape backward_shape(int64_t D, bool wide, int vec)
{
    if (wide) {
        for (int t = 4; t <= 16; t *= 2)
            if (D <= t * vec) return {t, vec, 128};
        for (int c = vec; c <= 32; c += vec)
            if (D <= 32 * c) return {32, c, 128};
        return {D <= 4096 ? 128 : 256, 32, D <= 4096 ? 128 : 256};
    }
    for (int t = 8; t <= 32; t *= 2)
        if (D <= 4 * t) return {t, 4, 128};
    if (D <= 512) return {32, 16, 128};
    return D <= 2048 ? BackwardShape{128, 16, 128} : BackwardShape{512, 16, 512};
}

constexpr int64_t kMostColumns = 8192;  // of rows held in registers

bool backward_wide(const NormArgs &a, int64_t size) { return a.ldx * size % 16 == 0 && a.lddy * size % 16 == 0 && aligned(a.x, 16) && aligned(a.dy, 16); }

// Blocks whose sums meet in the workspace; the same for every alignment, so that the workspace does not depend on it.
int backward_blocks(int64_t R, int64_t D)
{
    if (D > kMostColumns) {
        const int64_t chunks = (R + 63) / 64;
        return static_cast<int>(chunks < 64 ? chunks : 64);
    }
    const int64_t rows = D <= 32 ? 16 : D <= 1024 ? 4 : 1;  // a block's rows, at least
    const int64_t blocks = (R + rows - 1) / rows, most = D <= 4096 ? 444 : 222;
    return static_cast<int>(blocks < most ? blocks : most);
}

template <class T, int TPR, int VPT, bool WIDE, int NT> int backward_with(const NormArgs &a, int blocks, cudaStream_t s)
{
    auto *kernel = a.param_type == SPDY_F32 ? norm_backward_kernel<T, float, TPR, VPT, WIDE, WIDE, NT> : norm_backward_kernel<T, T, TPR, VPT, WIDE, WIDE, NT>;
    const size_t smem = a.want_params ? static_cast<size_t>(NT / TPR - 1) * 2 * static_cast<size_t>(a.D) * sizeof(float) : 0;
    if (smem > 32 * 1024) SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    kernel<<<blocks, NT, smem, s>>>(a);
    return finish_launch();
}

template <class T> int backward(const NormArgs &a, int blocks, cudaStream_t s)
{
    if (a.D > kMostColumns) {
        if (a.R > 0x7fffffff) return SPDY_ERR_UNSUPPORTED;
        // the columns first: dx may overwrite dy or x
        if (a.want_params) {
            norm_backward_columns_kernel<T><<<dim3(static_cast<unsigned>((a.D + 255) / 256), static_cast<unsigned>(blocks)), 256, 0, s>>>(a, (a.R + blocks - 1) / blocks);
            const int rc = finish_launch();
            if (rc != SPDY_OK) return rc;
        }
        norm_backward_long_kernel<T, 512><<<static_cast<unsigned>(a.R), 512, 0, s>>>(a);
        return finish_launch();
    }
    constexpr int VEC = Elem<T>::kVec;
    const bool wide = backward_wide(a, sizeof(T));
    const BackwardShape p = backward_shape(a.D, wide, VEC);
    if (wide) {
        if (p.threads == 4) return backward_with<T, 4, 1, true, 128>(a, blocks, s);
        if (p.threads == 8) return backward_with<T, 8, 1, true, 128>(a, blocks, s);
        if (p.threads == 16) return backward_with<T, 16, 1, true, 128>(a, blocks, s);
        if (p.threads == 128) return backward_with<T, 128, 32 / VEC, true, 128>(a, blocks, s);
        if (p.threads == 256) return backward_with<T, 256, 32 / VEC, true, 256>(a, blocks, s);
        if (p.columns <= 8) return backward_with<T, 32, 8 / VEC, true, 128>(a, blocks, s);
        if (p.columns <= 16) return backward_with<T, 32, 16 / VEC, true, 128>(a, blocks, s);
        if (p.columns <= 24) return backward_with<T, 32, 24 / VEC, true, 128>(a, blocks, s);
        return backward_with<T, 32, 32 / VEC, true, 128>(a, blocks, s);
    }
    if (p.threads == 8) return backward_with<T, 8, 4, false, 128>(a, blocks, s);
    if (p.threads == 16) return backward_with<T, 16, 4, false, 128>(a, blocks, s);
    if (p.threads == 128) return backward_with<T, 128, 16, false, 128>(a, blocks, s);
    if (p.threads == 512) return backward_with<T, 512, 16, false, 512>(a, blocks, s);
    if (p.columns <= 4) return backward_with<T, 32, 4, false, 128>(a, blocks, s);
    return backward_with<T, 32, 16, false, 128>(a, blocks, s);
}

constexpr int64_t kMostWidth = 0x7fffffff - 64;

bool matrix_ok(const void *p, int64_t ld, int dtype, int64_t R, int64_t D) { return ld >= D && (R == 0 || D == 0 || (p && aligned(p, type_size(dtype)))); }
bool params_ok(const void *p, int type, int dtype) { return !p || ((type == dtype || type == SPDY_F32) && aligned(p, type_size(type))); }

}  // namespace

extern "C" {

int spdy_layer_norm(const void *x, int64_t ldx, int dtype, const void *weight, const void *bias, int param_dtype, int64_t R, int64_t D, float eps, void *y,
                    int64_t ldy, float *mean, float *rstd, void *cuda_stream)
{
    if (!known_type(dtype) || R < 0 || D < 1 || D > kMostWidth || !(eps >= 0.f && eps <= 3.4e38f) || !matrix_ok(x, ldx, dtype, R, D) ||
        !matrix_ok(y, ldy, dtype, R, D) || !params_ok(weight, param_dtype, dtype) || !params_ok(bias, param_dtype, dtype))
        return SPDY_ERR_INVALID_ARG;
    if (R == 0) return SPDY_OK;
    NormArgs a = {};
    a.x = x, a.ldx = ldx, a.weight = weight, a.bias = bias, a.param_type = param_dtype, a.R = R, a.D = D, a.eps = eps;
    a.y = y, a.ldy = ldy, a.mean = mean, a.rstd = rstd;
    a.params_wide = (aligned(weight, 16) ? 1 : 0) | (aligned(bias, 16) ? 2 : 0);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return dtype == SPDY_F32 ? forward<float>(a, s) : dtype == SPDY_BF16 ? forward<__nv_bfloat16>(a, s) : forward<__half>(a, s);
}

size_t spdy_layer_norm_backward_workspace_bytes(int64_t R, int64_t D, int dtype)
{
    if (R <= 0 || D <= 0 || D > kMostWidth || !known_type(dtype)) return 0;
    return static_cast<size_t>(backward_blocks(R, D)) * 2 * static_cast<size_t>(D) * sizeof(float);
}

int spdy_layer_norm_backward(const void *dy, int64_t lddy, const void *x, int64_t ldx, int dtype, const void *weight, int param_dtype, const float *mean,
                             const float *rstd, int64_t R, int64_t D, void *dx, int64_t lddx, float *dweight, float *dbias, void *workspace,
                             size_t workspace_bytes, void *cuda_stream)
{
    if (!known_type(dtype) || R < 0 || D < 1 || D > kMostWidth || !matrix_ok(dy, lddy, dtype, R, D) || !matrix_ok(x, ldx, dtype, R, D) ||
        !matrix_ok(dx, lddx, dtype, R, D) || !params_ok(weight, param_dtype, dtype) || (R > 0 && (!mean || !rstd)))
        return SPDY_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (R == 0) {
        if (dweight) SPDY_EVAL_TRY(cudaMemsetAsync(dweight, 0, static_cast<size_t>(D) * sizeof(float), s));
        if (dbias) SPDY_EVAL_TRY(cudaMemsetAsync(dbias, 0, static_cast<size_t>(D) * sizeof(float), s));
        return SPDY_OK;
    }
    NormArgs a = {};
    a.dy = dy, a.lddy = lddy, a.x = x, a.ldx = ldx, a.weight = weight, a.param_type = param_dtype, a.R = R, a.D = D;
    a.dx = dx, a.lddx = lddx, a.in_mean = mean, a.in_rstd = rstd;
    a.want_params = dweight || dbias;
    a.params_wide = aligned(weight, 16) ? 1 : 0;
    if (a.want_params) {
        if (!workspace || !aligned(workspace, 256)) return SPDY_ERR_INVALID_ARG;
        if (workspace_bytes < spdy_layer_norm_backward_workspace_bytes(R, D, dtype)) return SPDY_ERR_WORKSPACE_TOO_SMALL;
        a.partial = static_cast<float *>(workspace);
    }
    const int blocks = backward_blocks(R, D);
    const int rc = dtype == SPDY_F32 ? backward<float>(a, blocks, s) : dtype == SPDY_BF16 ? backward<__nv_bfloat16>(a, blocks, s) : backward<__half>(a, blocks, s);
    if (rc != SPDY_OK || !a.want_params) return rc;
    norm_columns_kernel<<<static_cast<unsigned>((D + 31) / 32 * 2), 1024, 0, s>>>(a.partial, blocks, D, dweight, dbias);
    return finish_launch();
}

}  // extern "C"
