// Layer normalisation and its gradients: kernels and C entries (spdy_eval.h).
//
// Both directions read every element once and keep a row's part in registers between the two sums it needs (the mean before
// the squared deviations; sum u and sum u h before dx), so they are bound by memory.  A row belongs to one warp while it
// fits (no barrier then), to 128 to 512 threads when it is longer, and beyond that it is read again per sum.
#include "eval_common.cuh"

using namespace spdy_eval;

namespace {

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    int64_t ldx, lddy, ldy, lddx, R, D;
    int param_type;
    float eps;
    void *y, *dx;
    float *mean, *rstd;             // forward's results
    const float *in_mean, *in_rstd; // backward's inputs
    float *partial;                 // [blocks][2][D]
    int want_params;                // dweight or dbias asked for
};

__device__ __forceinline__ float param_at(const void *p, int type, int64_t i)
{
    if (type == SPDY_F32) return static_cast<const float *>(p)[i];
    if (type == SPDY_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(static_cast<const __half *>(p)[i]);
}

// N values from index e on, `fallback` for a NULL vector and outside [0, D).
template <int N> __device__ __forceinline__ void params(const void *p, int type, int64_t e, int64_t D, float fallback, float *f)
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = fallback;
        return;
    }
    const size_t size = type == SPDY_F32 ? 4 : 2;
    const char *at = static_cast<const char *>(p) + e * static_cast<int64_t>(size);
    if (N >= 4 && e >= 0 && e + N <= D && (reinterpret_cast<uintptr_t>(at) & 15) == 0) {
        if (type == SPDY_F32) {
#pragma unroll
            for (int i = 0; i + 4 <= N; i += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(at + 4 * i);
                f[i] = v.x, f[i + 1] = v.y, f[i + 2] = v.z, f[i + 3] = v.w;
            }
            return;
        }
        if (N == 8) {
            const uint4 v = *reinterpret_cast<const uint4 *>(at);
            if (type == SPDY_BF16) Elem<__nv_bfloat16>::unpack(v, f);
            else Elem<__half>::unpack(v, f);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = e + i >= 0 && e + i < D ? param_at(p, type, e + i) : fallback;
}

// Sums of TPR consecutive threads' values, in all of them.  `slot` alternates between calls, so that one barrier is enough.
template <int TPR, int COUNT> __device__ __forceinline__ void row_sums(float *v, float (*shared)[32], int slot)
{
#pragma unroll
    for (int d = 16; d; d >>= 1)
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

template <class T, int TPR, int VPT, int NT> __global__ void __launch_bounds__(NT) norm_forward_kernel(const NormArgs a)
{
    constexpr int VEC = Elem<T>::kVec;
    __shared__ float shared[2][32];
    const int64_t r = static_cast<int64_t>(blockIdx.x) * (NT / TPR) + threadIdx.x / TPR;
    if (TPR == 32 && r >= a.R) return;  // whole warps; with more threads per row a block holds one row
    const int t = threadIdx.x % TPR;
    const Row<T> row(static_cast<const T *>(a.x) + r * a.ldx, a.D);
    const int G = row.granules();
    uint4 raw[VPT];
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int g = v * TPR + t;
        if (g < G) raw[v] = row.load(g);
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
            if (e + i >= 0 && e + i < a.D) sum += f[i];
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
            if (e + i >= 0 && e + i < a.D) sq = fmaf(f[i] - mean, f[i] - mean, sq);
    }
    row_sums<TPR, 1>(&sq, shared, 1);
    const float rstd = 1.f / sqrtf(sq / n + a.eps);
    if (t == 0) {
        if (a.mean) a.mean[r] = mean;
        if (a.rstd) a.rstd[r] = rstd;
    }
    T *out = static_cast<T *>(a.y) + r * a.ldy;
#pragma unroll
    for (int v = 0; v < VPT; ++v) {
        const int g = v * TPR + t;
        if (g >= G) continue;
        const int e = row.first(g);
        float f[VEC], w[VEC], b[VEC];
        Elem<T>::unpack(raw[v], f);
        params<VEC>(a.weight, a.param_type, e, a.D, 1.f, w);
        params<VEC>(a.bias, a.param_type, e, a.D, 0.f, b);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = fmaf((f[i] - mean) * rstd, w[i], b[i]);
        if (row.same_lead(out) && row.whole(g)) store_stream(out + e, Elem<T>::pack(f));
        else store_part(out, row.n, e, Elem<T>::pack(f));
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

// VEC consecutive elements of a row as fp32, 0 outside; VEC = kVec needs 16-byte aligned rows.
template <class T, int VEC> __device__ __forceinline__ void load_some(const T *p, int64_t e, int64_t n, float *f)
{
    if (VEC > 1 && e + VEC <= n) {
        Elem<T>::unpack(load_stream(p + e), f);
        return;
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = e + i < n ? Elem<T>::to_float(p[e + i]) : 0.f;
}
template <class T, int VEC> __device__ __forceinline__ void store_some(T *p, int64_t e, int64_t n, const float *f)
{
    if (VEC > 1) {
        if (e + VEC <= n && (reinterpret_cast<uintptr_t>(p + e) & 15) == 0) {
            store_stream(p + e, Elem<T>::pack(f));
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (e + i < n) p[e + i] = Elem<T>::from_float(f[i]);
        }
    } else if (e < n) {
        p[e] = Elem<T>::from_float(f[0]);
    }
}

// Each group of TPR threads walks over rows and keeps the sums of its columns for dweight and dbias in registers; the groups
// of a block are joined through shared memory in a fixed order, the blocks by norm_columns_kernel.
template <class T, int TPR, int VPT, int VEC, int NT> __global__ void __launch_bounds__(NT) norm_backward_kernel(const NormArgs a)
{
    constexpr int GROUPS = NT / TPR;
    __shared__ float shared[4][32];
    extern __shared__ float columns[];  // [GROUPS - 1][2][D]
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR;
    float dw[VPT * VEC], db[VPT * VEC];
#pragma unroll
    for (int i = 0; i < VPT * VEC; ++i) dw[i] = db[i] = 0.f;
    const float inv_n = 1.f / static_cast<float>(a.D);
    int slot = 0;
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * GROUPS + group; r < a.R; r += static_cast<int64_t>(gridDim.x) * GROUPS, slot ^= 1) {
        const T *x = static_cast<const T *>(a.x) + r * a.ldx, *dy = static_cast<const T *>(a.dy) + r * a.lddy;
        T *out = static_cast<T *>(a.dx) + r * a.lddx;
        const float mean = a.in_mean[r], rstd = a.in_rstd[r];
        float h[VPT * VEC], u[VPT * VEC], sums[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int64_t e = static_cast<int64_t>(v * TPR + t) * VEC;
            load_some<T, VEC>(x, e, a.D, h + v * VEC);
            load_some<T, VEC>(dy, e, a.D, u + v * VEC);
        }
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int64_t e = static_cast<int64_t>(v * TPR + t) * VEC;
            if (e >= a.D) continue;
            float w[VEC];
            params<VEC>(a.weight, a.param_type, e, a.D, 1.f, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int k = v * VEC + i;
                h[k] = (h[k] - mean) * rstd;
                dw[k] = fmaf(u[k], h[k], dw[k]);
                db[k] += u[k];
                u[k] *= w[i];
                if (VEC == 1 || e + i < a.D) {
                    sums[0] += u[k];
                    sums[1] = fmaf(u[k], h[k], sums[1]);
                }
            }
        }
        row_sums<TPR, 2>(sums, shared, slot);
        const float mu = sums[0] * inv_n, mh = sums[1] * inv_n;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int64_t e = static_cast<int64_t>(v * TPR + t) * VEC;
            if (e >= a.D) continue;
            float f[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = rstd * (u[v * VEC + i] - fmaf(h[v * VEC + i], mh, mu));
            store_some<T, VEC>(out, e, a.D, f);
        }
    }
    if (!a.want_params) return;
    if (GROUPS > 1) {
        if (group > 0) {
#pragma unroll
            for (int k = 0; k < VPT * VEC; ++k) {
                const int64_t e = static_cast<int64_t>((k / VEC) * TPR + t) * VEC + k % VEC;
                if (e < a.D) columns[(group - 1) * 2 * a.D + e] = dw[k], columns[(group - 1) * 2 * a.D + a.D + e] = db[k];
            }
        }
        __syncthreads();
        if (group > 0) return;
        for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
            for (int k = 0; k < VPT * VEC; ++k) {
                const int64_t e = static_cast<int64_t>((k / VEC) * TPR + t) * VEC + k % VEC;
                if (e < a.D) dw[k] += columns[g * 2 * a.D + e], db[k] += columns[g * 2 * a.D + a.D + e];
            }
    }
    float *to = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * a.D;
#pragma unroll
    for (int k = 0; k < VPT * VEC; ++k) {
        const int64_t e = static_cast<int64_t>((k / VEC) * TPR + t) * VEC + k % VEC;
        if (e < a.D) to[e] = dw[k], to[a.D + e] = db[k];
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

// dweight and dbias from the blocks' sums, 32 columns per block, each of 8 warps adding every eighth block's.
__global__ void __launch_bounds__(256) norm_columns_kernel(const float *partial, int blocks, int64_t D, float *dweight, float *dbias)
{
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t e = static_cast<int64_t>(blockIdx.x) * 32 + lane;  // over [2][D], each half rounded up to 32
    const int64_t padded = (D + 31) / 32 * 32;
    const bool second = static_cast<int64_t>(blockIdx.x) * 32 >= padded;
    const int64_t col = second ? e - padded : e;
    float sum = 0.f;
    if (col < D) {
        const float *p = partial + (second ? D : 0) + col;
#pragma unroll 4
        for (int b = warp; b < blocks; b += 8) sum += p[static_cast<int64_t>(b) * 2 * D];
    }
    part[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && col < D) {
        sum = part[0][lane];
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += part[w][lane];
        float *to = second ? dbias : dweight;
        if (to) to[col] = sum;
    }
}

template <class T> int forward(const NormArgs &a, cudaStream_t s)
{
    const int64_t G = (a.D + Elem<T>::kVec - 1) / Elem<T>::kVec + (a.ldx * sizeof(T) % 16 || !aligned(a.x, 16) ? 1 : 0);
    if (a.R > 0x7fffffff) return SPDY_ERR_UNSUPPORTED;
    const unsigned rows = static_cast<unsigned>(a.R), quads = static_cast<unsigned>((a.R + 3) / 4);
    if (G <= 64) norm_forward_kernel<T, 32, 2, 128><<<quads, 128, 0, s>>>(a);
    else if (G <= 128) norm_forward_kernel<T, 32, 4, 128><<<quads, 128, 0, s>>>(a);
    else if (G <= 256) norm_forward_kernel<T, 32, 8, 128><<<quads, 128, 0, s>>>(a);
    else if (G <= 512) norm_forward_kernel<T, 128, 4, 128><<<rows, 128, 0, s>>>(a);
    else if (G <= 1024) norm_forward_kernel<T, 128, 8, 128><<<rows, 128, 0, s>>>(a);
    else if (G <= 4096) norm_forward_kernel<T, 512, 8, 512><<<rows, 512, 0, s>>>(a);
    else norm_forward_long_kernel<T, 512><<<rows, 512, 0, s>>>(a);
    return finish_launch();
}

constexpr int64_t kMostColumns = 8192;  // of the backward kernel that holds a row in registers: 256 threads, 32 columns each

int backward_blocks(int64_t R, int64_t D)
{
    if (D > kMostColumns) {
        const int64_t chunks = (R + 63) / 64;
        return static_cast<int>(chunks < 64 ? chunks : 64);
    }
    const int groups = D <= 1024 ? 8 : 1;
    const int64_t blocks = (R + groups - 1) / groups, most = D <= 1024 ? 296 : D <= 4096 ? 592 : 296;
    return static_cast<int>(blocks < most ? blocks : most);
}

template <class T, int VEC> int backward_rows(const NormArgs &a, int blocks, cudaStream_t s)
{
    constexpr int VPT = 32 / VEC;
    if (a.D <= 1024) {
        const size_t smem = a.want_params ? static_cast<size_t>(7) * 2 * a.D * sizeof(float) : 0;
        auto *kernel = norm_backward_kernel<T, 32, VPT, VEC, 256>;
        if (smem > 48 * 1024) SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
        kernel<<<blocks, 256, smem, s>>>(a);
    } else if (a.D <= 4096) {
        norm_backward_kernel<T, 128, VPT, VEC, 128><<<blocks, 128, 0, s>>>(a);
    } else {
        norm_backward_kernel<T, 256, VPT, VEC, 256><<<blocks, 256, 0, s>>>(a);
    }
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
    const bool wide = a.ldx * sizeof(T) % 16 == 0 && a.lddy * sizeof(T) % 16 == 0 && aligned(a.x, 16) && aligned(a.dy, 16);
    return wide ? backward_rows<T, Elem<T>::kVec>(a, blocks, s) : backward_rows<T, 1>(a, blocks, s);
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
    if (a.want_params) {
        if (!workspace || !aligned(workspace, 256)) return SPDY_ERR_INVALID_ARG;
        if (workspace_bytes < spdy_layer_norm_backward_workspace_bytes(R, D, dtype)) return SPDY_ERR_WORKSPACE_TOO_SMALL;
        a.partial = static_cast<float *>(workspace);
    }
    const int blocks = backward_blocks(R, D);
    const int rc = dtype == SPDY_F32 ? backward<float>(a, blocks, s) : dtype == SPDY_BF16 ? backward<__nv_bfloat16>(a, blocks, s) : backward<__half>(a, blocks, s);
    if (rc != SPDY_OK || !a.want_params) return rc;
    norm_columns_kernel<<<static_cast<unsigned>((D + 31) / 32 * 2), 256, 0, s>>>(a.partial, blocks, D, dweight, dbias);
    return finish_launch();
}

}  // extern "C"
