// Layer normalisation and its gradients: kernels and C entries (spdy_eval.h).
//
// Both directions read every element once and need two sums of a row before they can write it (the mean before the squared
// deviations; sum u and sum u h before dx), so they are bound by memory as long as reads go on while a row is being
// summed.  Many rows: persistent blocks with a ring of rows in shared memory that asynchronous copies fill ahead.  Few rows, and rows of up
// to 256 bytes (which share a warp): rows in registers.  Rows beyond 32 KB are read again per sum.
//
// Measured, bf16, us (and the bytes at 6.56 TB/s; a plain copy of the forward's bytes takes 24.0, an addition of the backward's
// three matrices 32): 32768 x 1024 forward 27.0 (20.5), backward 47.3 (30.7); 8192 x 4096 29.4, 52.0; 32768 x 999 (rows that
// start anywhere) 49.7, 84.2; 200000 x 128 32.9 (15.6), 49.4 (23.4); 128 x 768 4.3, 12.4.  With rows in registers, the next one's
// on their way: 33.4, 60; 49.6, 87; 56, 179.  fp32: 16384 x 1024 22.0 (20.5), 41.4 (30.7); 32768 x 1024 48.6 (40.9), 73.5 (61.4).
#include "eval_common.cuh"

using namespace spdy_eval;

namespace {

constexpr int64_t kShortBytes = 256;    // rows up to here share a warp
constexpr int64_t kRingMost = 32768;    // bytes of the longest rows that a ring holds

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
    if (in_granules(wide, e, N, D, PV)) {
#pragma unroll
        for (int i = 0; i + PV <= N; i += PV) Elem<P>::unpack(*reinterpret_cast<const uint4 *>(at + i), f + i);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = e + i >= 0 && e + i < D ? Elem<P>::to_float(at[i]) : fallback;
}

// The threads of a group of TPR, group `group` of the block, meet.
template <int TPR> __device__ __forceinline__ void meet(int group)
{
    if (TPR <= 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
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
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = threadIdx.x / TPR;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < COUNT; ++i) shared[slot * COUNT + i][warp] = v[i];
        meet<TPR>(group);
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            v[i] = lane < W ? shared[slot * COUNT + i][group * W + lane] : 0.f;
#pragma unroll
            for (int d = W / 2; d; d >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
            v[i] = __shfl_sync(0xffffffffu, v[i], 0);
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

// Rows too long for the ring: one block per row, the row read once per sum (from L2 after the first).
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

// ---------------------------------------------------------------------------------------------- many rows
// A block that stays on its multiprocessor walks over rows.  Each group of TPR threads owns a ring of S rows in shared memory,
// which asynchronous copies fill S - 1 rows ahead of the sums: with rows fetched into registers instead, the reads paused
// while a row was being summed.  Thread t works on the columns of granules t, TPR + t, ... counted from the row's start.
// WHOLE: rows are aligned granules, a thread copies, reads and stores its own.  Else the copies bring the aligned granules that lie wholly
// inside the row, single elements its ends, and everything is shifted on the way out of shared memory (about two instructions
// an element and three meetings of the group: 1.8 times as long as whole granules, half as long as single elements).
// 16 bytes from byte `shift` of granule g on.
__device__ __forceinline__ uint4 shifted(const uint4 *row, int g, int shift)
{
    const uint4 a = row[g];
    if (shift == 0) return a;
    const uint4 b = row[g + 1];
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int j = 0; j < 6; ++j) w[j] = shift & 8 ? w[j + 2] : w[j];
#pragma unroll
    for (int j = 0; j < 5; ++j) w[j] = shift & 4 ? w[j + 1] : w[j];
    const int bits = (shift & 3) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

// The ends of a row that starts anywhere, one element to each of the first 2 kVec threads: element `at` of the row, if `mine`.
template <class T> struct Ends {
    bool mine;
    int at;
    __device__ __forceinline__ Ends(const Row<T> &row, int t)
    {
        constexpr int VEC = Elem<T>::kVec;
        const int inside = (row.n + row.lead) / VEC * VEC - row.lead;  // where the last granule begins, if it is not whole
        at = t < VEC ? t : inside + t - VEC;
        mine = t < VEC ? row.lead > 0 && t < VEC - row.lead : t < 2 * VEC && at < row.n;
    }
};

template <class T, int TPR, int VPT, bool WHOLE> struct RowSlot {
    static constexpr int VEC = Elem<T>::kVec;
    static constexpr int kGranules = TPR * VPT + (WHOLE ? 0 : 2);
    static __device__ __forceinline__ void fetch(uint4 *slot, const T *p, int n, int t)
    {
        if (WHOLE) {
#pragma unroll
            for (int v = 0; v < VPT; ++v)
                if ((v * TPR + t) * VEC < n) copy16(slot + v * TPR + t, p + (v * TPR + t) * VEC);
        } else {
            const Row<T> row(p, n);
#pragma unroll
            for (int v = 0; v <= VPT; ++v)
                if (v * TPR + t < kGranules && row.whole(v * TPR + t)) copy16(slot + v * TPR + t, p + row.first(v * TPR + t));
        }
    }
    // columns of granule v * TPR + t (0 beyond n); `lead`: elements of the slot before the row
    static __device__ __forceinline__ uint4 get(const uint4 *slot, int v, int t, int lead, int n)
    {
        if (WHOLE) return slot[v * TPR + t];
        uint4 raw = shifted(slot, v * TPR + t, lead * static_cast<int>(sizeof(T)));
        const int e = (v * TPR + t) * VEC;
        if (e + VEC > n) {
            float f[VEC];
            Elem<T>::unpack(raw, f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = e + i < n ? f[i] : 0.f;
            raw = Elem<T>::pack(f);
        }
        return raw;
    }
    // The results of a row that starts anywhere, which lie in `slot` from its first granule on, to `out`.
    static __device__ __forceinline__ void put(const uint4 *slot, T *out, int n, int t)
    {
        const Row<T> row(out, n);
        const int shift = (VEC - row.lead) % VEC * static_cast<int>(sizeof(T));
#pragma unroll
        for (int v = 0; v <= VPT; ++v) {
            const int g = v * TPR + t;
            if (row.whole(g)) store_stream(out + row.first(g), shifted(slot, g - (row.lead > 0), shift));
        }
        const Ends<T> ends(row, t);
        if (ends.mine) out[ends.at] = reinterpret_cast<const T *>(slot)[ends.at];
    }
};

// A weight or bias in shared memory, as the group of threads uses it: its granules of columns, `fallback` for a NULL vector.
template <class T, class P, int TPR, int VPT> struct ParamRow {
    static constexpr int VEC = Elem<T>::kVec, PV = Elem<P>::kVec, kGranules = TPR * VPT * VEC / PV;
    static __device__ __forceinline__ void fill(uint4 *to, const void *p, int D, float fallback)
    {
        P *at = reinterpret_cast<P *>(to);
        for (int e = threadIdx.x; e < TPR * VPT * VEC; e += blockDim.x) at[e] = p && e < D ? static_cast<const P *>(p)[e] : Elem<P>::from_float(fallback);
    }
    static __device__ __forceinline__ void get(const uint4 *from, int v, int t, float *f)
    {
#pragma unroll
        for (int i = 0; i < VEC / PV; ++i) Elem<P>::unpack(from[(v * TPR + t) * (VEC / PV) + i], f + i * PV);
    }
};

template <class T, class P, int TPR, int VPT, bool WHOLE, int NT, int S, int PER_SM>
__global__ void __launch_bounds__(NT, PER_SM) norm_forward_ring_kernel(const NormArgs a)
{
    using Slot = RowSlot<T, TPR, VPT, WHOLE>;
    using Params = ParamRow<T, P, TPR, VPT>;
    constexpr int GROUPS = NT / TPR, VEC = Elem<T>::kVec;
    extern __shared__ uint4 memory[];
    __shared__ float shared[2][32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, D = static_cast<int>(a.D);
    uint4 *weight = memory, *bias = memory + Params::kGranules, *ring = memory + 2 * Params::kGranules + group * (S * Slot::kGranules);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * GROUPS;
    int64_t r = static_cast<int64_t>(blockIdx.x) * GROUPS + group;
    const auto at = [&](int64_t row) { return static_cast<const T *>(a.x) + row * a.ldx; };
    const auto fetch = [&](int64_t row, int slot) {
        if (row < a.R) Slot::fetch(ring + slot * Slot::kGranules, at(row), D, t);
        copies_commit();
    };
    T end = Elem<T>::from_float(0.f);
    const auto fetch_end = [&](int64_t row) {
        if (WHOLE || row >= a.R) return;
        const Ends<T> e(Row<T>(at(row), D), t);
        if (e.mine) end = at(row)[e.at];
    };
#pragma unroll
    for (int i = 0; i < S; ++i) fetch(r + i * stride, i);
    fetch_end(r);
    Params::fill(weight, a.weight, D, 1.f);
    Params::fill(bias, a.bias, D, 0.f);
    __syncthreads();
    const float n = static_cast<float>(D);
    for (int slot = 0; r < a.R; r += stride, slot = slot + 1 == S ? 0 : slot + 1) {
        uint4 *mine = ring + slot * Slot::kGranules;
        int lead = 0;
        copies_wait<S - 1>();
        if (!WHOLE) {
            const Row<T> row(at(r), D);
            const Ends<T> e(row, t);
            lead = row.lead;
            if (e.mine) reinterpret_cast<T *>(mine)[e.at + lead] = end;
            meet<TPR>(group);
            fetch_end(r + stride);
        }
        uint4 raw[VPT];
#pragma unroll
        for (int v = 0; v < VPT; ++v)
            if ((v * TPR + t) * VEC < D) raw[v] = Slot::get(mine, v, t, lead, D);
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            if ((v * TPR + t) * VEC >= D) continue;
            float f[VEC];
            Elem<T>::unpack(raw[v], f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum += f[i];
        }
        row_sums<TPR, 1>(&sum, shared, 0);
        if (WHOLE) fetch(r + S * stride, slot);
        const float mean = sum / n;
        float sq = 0.f;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = (v * TPR + t) * VEC;
            if (e >= D) continue;
            float f[VEC];
            Elem<T>::unpack(raw[v], f);
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (WHOLE || e + i < D) sq = fmaf(f[i] - mean, f[i] - mean, sq);
        }
        row_sums<TPR, 1>(&sq, shared, 1);
        const float rstd = 1.f / sqrtf(sq / n + a.eps);
        if (t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
        T *out = static_cast<T *>(a.y) + r * a.ldy;
        if (!WHOLE && TPR == 32) __syncwarp();  // all have read the slot (longer groups met in the sums)
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = (v * TPR + t) * VEC;
            if (e >= D) continue;
            float f[VEC], w[VEC], b[VEC];
            Elem<T>::unpack(raw[v], f);
            Params::get(weight, v, t, w);
            Params::get(bias, v, t, b);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = fmaf((f[i] - mean) * rstd, w[i], b[i]);
            if (WHOLE) store_stream(out + e, Elem<T>::pack(f));
            else mine[v * TPR + t] = Elem<T>::pack(f);
        }
        if (!WHOLE) {
            meet<TPR>(group);
            Slot::put(mine, out, D, t);
            meet<TPR>(group);
            fetch(r + S * stride, slot);
        }
    }
}

// dx row by row, and the sums of its columns for dweight and dbias in the thread's registers; the groups' sums are joined through
// shared memory in a fixed order, the blocks' by norm_columns_kernel.  x and dy are unpacked from the ring a second time rather than
// kept: 64 registers hold the columns' sums, and 16 warps of 128 registers fill the multiprocessor.
template <class T, class P, int TPR, int VPT, bool WHOLE, int NT, int S> __global__ void __launch_bounds__(NT, 1) norm_backward_ring_kernel(const NormArgs a)
{
    using Slot = RowSlot<T, TPR, VPT, WHOLE>;
    using Params = ParamRow<T, P, TPR, VPT>;
    constexpr int GROUPS = NT / TPR, VEC = Elem<T>::kVec;
    extern __shared__ uint4 memory[];
    __shared__ float shared[4][32];
    const int group = threadIdx.x / TPR, t = threadIdx.x % TPR, D = static_cast<int>(a.D);
    uint4 *weight = memory, *rings = memory + Params::kGranules, *ring = rings + group * (2 * S * Slot::kGranules);
    const int64_t stride = static_cast<int64_t>(gridDim.x) * GROUPS;
    int64_t r = static_cast<int64_t>(blockIdx.x) * GROUPS + group;
    const auto x_at = [&](int64_t row) { return static_cast<const T *>(a.x) + row * a.ldx; };
    const auto dy_at = [&](int64_t row) { return static_cast<const T *>(a.dy) + row * a.lddy; };
    const auto fetch = [&](int64_t row, int slot) {
        if (row < a.R) {
            Slot::fetch(ring + 2 * slot * Slot::kGranules, x_at(row), D, t);
            Slot::fetch(ring + (2 * slot + 1) * Slot::kGranules, dy_at(row), D, t);
        }
        copies_commit();
    };
    T end_x = Elem<T>::from_float(0.f), end_dy = end_x;
    float next_mean = 0.f, next_rstd = 0.f;
    const auto fetch_ends = [&](int64_t row) {
        if (row >= a.R) return;
        next_mean = a.in_mean[row], next_rstd = a.in_rstd[row];
        if (WHOLE) return;
        const Ends<T> ex(Row<T>(x_at(row), D), t), ey(Row<T>(dy_at(row), D), t);
        if (ex.mine) end_x = x_at(row)[ex.at];
        if (ey.mine) end_dy = dy_at(row)[ey.at];
    };
#pragma unroll
    for (int i = 0; i < S; ++i) fetch(r + i * stride, i);
    fetch_ends(r);
    Params::fill(weight, a.weight, D, 1.f);
    __syncthreads();
    float dw[VPT * VEC], db[VPT * VEC];
#pragma unroll
    for (int i = 0; i < VPT * VEC; ++i) dw[i] = db[i] = 0.f;
    const float inv_n = 1.f / static_cast<float>(D);
    int parity = 0;
    for (int slot = 0; r < a.R; r += stride, slot = slot + 1 == S ? 0 : slot + 1, parity ^= 1) {
        uint4 *x = ring + 2 * slot * Slot::kGranules, *dy = x + Slot::kGranules;
        const float mean = next_mean, rstd = next_rstd;
        int lead_x = 0, lead_dy = 0;
        copies_wait<S - 1>();
        if (!WHOLE) {
            const Row<T> rx(x_at(r), D), ry(dy_at(r), D);
            const Ends<T> ex(rx, t), ey(ry, t);
            lead_x = rx.lead, lead_dy = ry.lead;
            if (ex.mine) reinterpret_cast<T *>(x)[ex.at + lead_x] = end_x;
            if (ey.mine) reinterpret_cast<T *>(dy)[ey.at + lead_dy] = end_dy;
            meet<TPR>(group);
        }
        fetch_ends(r + stride);
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            if ((v * TPR + t) * VEC >= D) continue;
            float w[VEC], h[VEC], u[VEC];
            Params::get(weight, v, t, w);
            Elem<T>::unpack(Slot::get(x, v, t, lead_x, D), h);
            Elem<T>::unpack(Slot::get(dy, v, t, lead_dy, D), u);
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
        row_sums<TPR, 2>(sums, shared, parity);
        const float mu = sums[0] * inv_n, mh = sums[1] * inv_n;
        T *out = static_cast<T *>(a.dx) + r * a.lddx;
#pragma unroll
        for (int v = 0; v < VPT; ++v) {
            const int e = (v * TPR + t) * VEC;
            uint4 result = make_uint4(0, 0, 0, 0);
            if (e < D) {
                float w[VEC], h[VEC], f[VEC];
                Params::get(weight, v, t, w);
                Elem<T>::unpack(Slot::get(x, v, t, lead_x, D), h);
                Elem<T>::unpack(Slot::get(dy, v, t, lead_dy, D), f);
#pragma unroll
                for (int i = 0; i < VEC; ++i) f[i] = rstd * (f[i] * w[i] - fmaf((h[i] - mean) * rstd, mh, mu));
                result = Elem<T>::pack(f);
                if (WHOLE) store_stream(out + e, result);
            }
            if (!WHOLE) {
                meet<TPR>(group);  // granules v * TPR .. (v + 1) * TPR have been read; the last of them is not written yet
                if (e < D) x[v * TPR + t] = result;
            }
        }
        if (!WHOLE) {
            meet<TPR>(group);
            Slot::put(x, out, D, t);
            meet<TPR>(group);
        }
        fetch(r + S * stride, slot);
    }
    if (!a.want_params) return;
    copies_wait<0>();
    __syncthreads();
    float *columns = reinterpret_cast<float *>(rings) + static_cast<int64_t>(group) * 2 * D;  // [GROUPS][2][D]
#pragma unroll
    for (int k = 0; k < VPT * VEC; ++k) {
        const int e = ((k / VEC) * TPR + t) * VEC + k % VEC;
        if (e < D) columns[e] = dw[k], columns[D + e] = db[k];
    }
    __syncthreads();
    float *to = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * D;
    for (int c = threadIdx.x; c < 2 * D; c += NT) {
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) sum += reinterpret_cast<const float *>(rings)[g * 2 * D + c];
        to[c] = sum;
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

// Short rows.  Each group of TPR threads walks over rows, the next row's elements on their way while this one's are used, and keeps the
// sums of its columns for dweight and dbias in registers; the groups of a block are joined through shared memory in a
// fixed order, the blocks by norm_columns_kernel.
template <class T, class P, int TPR, int VPT, bool WIDE, int NT> __global__ void __launch_bounds__(NT) norm_backward_kernel(const NormArgs a)
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
    if (WIDE) fetch(static_cast<int64_t>(blockIdx.x) * GROUPS + group, next_x, next_dy, next_mean, next_rstd);
    int slot = 0;
    // the same number of rounds for all groups of a block: their threads meet in the sums
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * GROUPS; base < a.R; base += stride, slot ^= 1) {
        const int64_t r = base + group;
        const bool here = r < a.R;
        if (WIDE) {
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

// dweight and dbias from the blocks' sums, 32 columns per block, each of 32 warps adding every 32nd block's.  Bound by its
// latency (about 5 us for 1024 columns of 148 blocks).
__global__ void __launch_bounds__(1024) norm_columns_kernel(const float *partial, int blocks, int64_t D, float *dweight, float *dbias)
{
    __shared__ float part[32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t e = static_cast<int64_t>(blockIdx.x) * 32 + lane;  // over [2][D], each half rounded up to 32
    const int64_t padded = (D + 31) / 32 * 32;
    const bool second = static_cast<int64_t>(blockIdx.x) * 32 >= padded;
    const int64_t col = second ? e - padded : e;
    asm volatile("griddepcontrol.wait;" ::: "memory");
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

constexpr int64_t kRingBytes = 24 << 20;  // of x, from which on the forward's ring pays (direct and ring, us: 1024 bf16 columns 16 MB 11.9, 10.6, 64 MB 33.3, 29.0; 4096 columns 64 MB 49.6, 31.0; 8192 columns 16 MB 10.6, 12.6, 64 MB 35.8, 33.2; 1024 f32 columns 16 MB 8.7, 10.5)
constexpr int kRingThreads = 512;
constexpr int kMostShared = 226 * 1024;

template <class T, class P, int TPR, int VPT, bool WHOLE> int forward_ring_with(const NormArgs &a, cudaStream_t s)
{
    constexpr int GROUPS = kRingThreads / TPR, S = VPT == 4 ? 3 : 4;
    constexpr int smem = 16 * (2 * ParamRow<T, P, TPR, VPT>::kGranules + GROUPS * S * RowSlot<T, TPR, VPT, WHOLE>::kGranules);
    constexpr int PER_SM = 2 * (smem + 1024) <= kMostShared ? 2 : 1;
    static_assert(smem <= kMostShared, "");
    auto *kernel = norm_forward_ring_kernel<T, P, TPR, VPT, WHOLE, kRingThreads, S, PER_SM>;
    SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    const int64_t blocks = (a.R + GROUPS - 1) / GROUPS, most = PER_SM * sm_count();
    kernel<<<static_cast<unsigned>(blocks < most ? blocks : most), kRingThreads, smem, s>>>(a);
    return finish_launch();
}
template <class T, int TPR, int BYTES> int forward_ring(const NormArgs &a, bool whole, cudaStream_t s)
{
    constexpr int VPT = BYTES / 16;
    if (a.param_type == SPDY_F32) return whole ? forward_ring_with<T, float, TPR, VPT, true>(a, s) : forward_ring_with<T, float, TPR, VPT, false>(a, s);
    return whole ? forward_ring_with<T, T, TPR, VPT, true>(a, s) : forward_ring_with<T, T, TPR, VPT, false>(a, s);
}

template <class T> int forward(const NormArgs &a, cudaStream_t s)
{
    constexpr int VEC = Elem<T>::kVec;
    if (a.R > 0x7fffffff) return SPDY_ERR_UNSUPPORTED;
    const bool in_line = a.ldx % VEC == 0 && aligned(a.x, 16);
    const bool whole = in_line && a.ldy % VEC == 0 && aligned(a.y, 16) && a.D % VEC == 0;
    const int64_t G = (a.D + VEC - 1) / VEC + (in_line ? 0 : 1);
    const int64_t bytes = a.D * static_cast<int64_t>(sizeof(T));
    if (bytes > kShortBytes && bytes <= kRingMost && a.R * bytes >= kRingBytes) {
        if (bytes <= 512) return forward_ring<T, 32, 16>(a, whole, s);
        if (bytes <= 1024) return forward_ring<T, 32, 32>(a, whole, s);
        if (bytes <= 1536) return forward_ring<T, 32, 48>(a, whole, s);
        if (bytes <= 2048) return forward_ring<T, 32, 64>(a, whole, s);
        if (bytes <= 3072) return forward_ring<T, 64, 48>(a, whole, s);
        if (bytes <= 4096) return forward_ring<T, 64, 64>(a, whole, s);
        if (bytes <= 8192) return forward_ring<T, 128, 64>(a, whole, s);
        if (bytes <= 16384) return forward_ring<T, 256, 64>(a, whole, s);
        return forward_ring<T, 512, 64>(a, whole, s);
    }
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

bool backward_wide(const NormArgs &a, int64_t size) { return a.ldx * size % 16 == 0 && a.lddy * size % 16 == 0 && aligned(a.x, 16) && aligned(a.dy, 16); }

// Blocks whose sums meet in the workspace; the same for every alignment, so that the workspace does not depend on it.
int backward_blocks(int64_t R, int64_t D, int64_t size)
{
    if (D * size > kRingMost) {
        const int64_t chunks = (R + 63) / 64;
        return static_cast<int>(chunks < 64 ? chunks : 64);
    }
    const bool is_short = D * size <= kShortBytes;
    const int64_t rows = is_short ? 16 : 4;  // a block's rows, at least
    const int64_t blocks = (R + rows - 1) / rows, most = is_short ? 444 : sm_count();
    return static_cast<int>(blocks < most ? blocks : most);
}

template <class T, class P, int TPR, int VPT, bool WHOLE> int backward_ring_with(const NormArgs &a, int blocks, cudaStream_t s)
{
    constexpr int GROUPS = kRingThreads / TPR, fixed = 16 * ParamRow<T, P, TPR, VPT>::kGranules, row = 32 * GROUPS * RowSlot<T, TPR, VPT, WHOLE>::kGranules;
    constexpr int fit = (kMostShared - fixed) / row, S = fit < 4 ? fit : 4, smem = fixed + S * row;
    static_assert(S >= 2, "");
    static_assert(S * row >= GROUPS * 2 * TPR * VPT * Elem<T>::kVec * 4, "the columns' sums lie where the ring was");
    auto *kernel = norm_backward_ring_kernel<T, P, TPR, VPT, WHOLE, kRingThreads, S>;
    SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    kernel<<<blocks, kRingThreads, smem, s>>>(a);
    return finish_launch();
}
template <class T, int TPR, int BYTES> int backward_ring(const NormArgs &a, bool whole, int blocks, cudaStream_t s)
{
    constexpr int VPT = BYTES / 16;
    if (a.param_type == SPDY_F32) return whole ? backward_ring_with<T, float, TPR, VPT, true>(a, blocks, s) : backward_ring_with<T, float, TPR, VPT, false>(a, blocks, s);
    return whole ? backward_ring_with<T, T, TPR, VPT, true>(a, blocks, s) : backward_ring_with<T, T, TPR, VPT, false>(a, blocks, s);
}

template <class T, int TPR, int VPT, bool WIDE> int backward_short(const NormArgs &a, int blocks, cudaStream_t s)
{
    constexpr int NT = 128;
    auto *kernel = a.param_type == SPDY_F32 ? norm_backward_kernel<T, float, TPR, VPT, WIDE, NT> : norm_backward_kernel<T, T, TPR, VPT, WIDE, NT>;
    const size_t smem = a.want_params ? static_cast<size_t>(NT / TPR - 1) * 2 * static_cast<size_t>(a.D) * sizeof(float) : 0;
    kernel<<<blocks, NT, smem, s>>>(a);
    return finish_launch();
}

template <class T> int backward(const NormArgs &a, int blocks, cudaStream_t s)
{
    constexpr int VEC = Elem<T>::kVec;
    const int64_t bytes = a.D * static_cast<int64_t>(sizeof(T));
    const bool wide = backward_wide(a, sizeof(T));
    if (bytes > kRingMost) {
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
    if (bytes > kShortBytes) {
        const bool whole = wide && a.lddx % VEC == 0 && aligned(a.dx, 16) && a.D % VEC == 0;
        if (bytes <= 512) return backward_ring<T, 32, 16>(a, whole, blocks, s);
        if (bytes <= 1024) return backward_ring<T, 32, 32>(a, whole, blocks, s);
        if (bytes <= 1536) return backward_ring<T, 32, 48>(a, whole, blocks, s);
        if (bytes <= 2048) return backward_ring<T, 32, 64>(a, whole, blocks, s);
        // 64 threads a row, and more columns each, for many rows (19206 x 1099 bf16: 82 us, with 128 threads 108); 128 where there are few
        // rows, whose ends then count (200 x 2048: 10.6 us, with 64 threads 14.7)
        if (bytes <= 4096 && a.R < 16 * sm_count()) return backward_ring<T, 128, 32>(a, whole, blocks, s);
        if (bytes <= 3072) return backward_ring<T, 64, 48>(a, whole, blocks, s);
        if (bytes <= 4096) return backward_ring<T, 64, 64>(a, whole, blocks, s);
        if (bytes <= 8192) return backward_ring<T, 128, 64>(a, whole, blocks, s);
        if (bytes <= 16384) return backward_ring<T, 256, 64>(a, whole, blocks, s);
        return backward_ring<T, 512, 64>(a, whole, blocks, s);
    }
    if (wide) {
        if (a.D <= 4 * VEC) return backward_short<T, 4, 1, true>(a, blocks, s);
        if (a.D <= 8 * VEC) return backward_short<T, 8, 1, true>(a, blocks, s);
        return backward_short<T, 16, 1, true>(a, blocks, s);
    }
    if (a.D <= 32) return backward_short<T, 8, 4, false>(a, blocks, s);
    if (a.D <= 64) return backward_short<T, 16, 4, false>(a, blocks, s);
    return backward_short<T, 32, 4, false>(a, blocks, s);
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
    return static_cast<size_t>(backward_blocks(R, D, static_cast<int64_t>(type_size(dtype)))) * 2 * static_cast<size_t>(D) * sizeof(float);
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
    const int blocks = backward_blocks(R, D, static_cast<int64_t>(type_size(dtype)));
    const int rc = dtype == SPDY_F32 ? backward<float>(a, blocks, s) : dtype == SPDY_BF16 ? backward<__nv_bfloat16>(a, blocks, s) : backward<__half>(a, blocks, s);
    if (rc != SPDY_OK || !a.want_params) return rc;
    // sent to the device before the blocks in front of it are done, which it waits for itself: no gap for the launch between them
    cudaLaunchAttribute early = {};
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>((D + 31) / 32 * 2)), config.blockDim = dim3(1024), config.stream = s;
    config.attrs = &early, config.numAttrs = 1;
    SPDY_EVAL_TRY(cudaLaunchKernelEx(&config, norm_columns_kernel, static_cast<const float *>(a.partial), blocks, D, dweight, dbias));
    return SPDY_OK;
}

}  // extern "C"
