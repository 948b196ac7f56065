// y = act(x w^T + bias) + residual: kernels and C entry (spdy_eval.h).
//
// The product runs on the tensor cores (tcgen05, 16-bit operands, fp32 accumulators in TMEM); one thread feeds it with TMA
// copies of 64-wide slices of x and w, one issues the matrix instructions, sixteen warps carry the finished tiles through the
// epilogue while the next tile is multiplied.  Large products pair two multiprocessors on a tile of 256 rows (cta_group::2), so
// that each brings half of the tile's rows of w: per product the pair moves 2/3 of what two single 128 x 256 tiles would
// (8192^3 with those: 1.29 PFLOP/s, with pairs 1.41 to 1.46, of 1.63 to 1.68 that the card's library product reaches).  Few rows (single tokens)
// are a matter of reading w once: a kernel of plain multiply-adds streams it.
//
// Measured, bf16, us in a graph (and the floor: the larger of bytes at 6.56 TB/s and operations at 1.68 PFLOP/s):
// 4096 x 768 x 3072 (rows, K, columns) with bias and gelu 23.0 (11.5), without 20.0, 16384 x 1024 x 4096 with gelu 105 (82), without 100,
// 8192 x 4096 x 1024 with residual 58 (41), 8192^3 713 to 755 (656), 512 x 1024 x 4096 12.7, 128 x 768 x 3072 9.4, 16 x 4096 x 1024 10.6.
// Bound: large products by the feed of the tensor cores (a stage's barriers and copies beside its products), the middle ones by whole rounds of tiles
// and the last one's epilogue, the small ones by the fixed way through barriers, TMEM and the exchange of parts (about 8 us).
#include "eval_tensor.cuh"

using namespace spdy_eval;

namespace spdy_eval {
int linear_logprobs_timeouts(cudaStream_t s, int *count);  // eval_linear_logprobs.cu
}

namespace {

namespace cg = cooperative_groups;

constexpr int kSlices = 2;                 // slices of a stage: a round of barriers costs about 400 cycles, the products of one slice 128 to 512
constexpr int kEpilogueWarps = 16;         // four to a scheduler: with two, a tile's epilogue took longer than its products at K = 768
constexpr int kThreads = 32 * (2 + kEpilogueWarps);
// At most this many rows take the multiply-add kernel.  It and the tensor cores in one build, us, with a w that comes from memory:
// 4096 x 4096 4 rows 11.2, 17.9, 8 rows 17.7, 18.0 to 22.5, 9 rows 23.7, 17.5; 1024 x 4096 8 rows 8.8, 8.8, 9 rows 11.9, 8.8; 768 x 768 8 rows
// 2.9, 6.4, 9 rows 3.1, 6.4; 2048 x 8192 4 rows 12.7, 19.1, 8 rows 20.9, 18.7.
constexpr int64_t kFewRows = 8;

struct LinearArgs {
    const void *x, *w, *bias, *residual;
    void *y;
    int64_t ldx, ldw, ldres, ldy, M, N, K;
    int dtype, bias_type, out_type, activation;
    int tiles_m, tiles_n, k_blocks;
    int wide_out, wide_res, wide_bias;     // 16-byte accesses are possible on every row of y, of residual, on bias
    int sectors, words;                    // every row of y and of the residual starts on 32 bytes; 16-bit rows of y start on 4
};

// ---------------------------------------------------------------------------------------------- epilogue
// 1 / x to about an ulp, on the special-function unit
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// z Phi(z), Phi the normal distribution function, as max(z, 0) - t Phi(-t) with t = |z|: Phi(-t) = exp(-t^2 / 2) E(t) keeps its
// leading digits however small it is (1/2 + erf / 2 would lose them from z = -2 on).  E falls slowly, like 1 / t in the end, and
// is s times a polynomial of degree 7 in s = 1 / (1 + 0.3 t) on 0 <= t <= 14 (least maximum of the relative error by reweighted
// least squares on Chebyshev nodes, 1.5e-7).  The result is within 8e-7 of itself for |z| < 4; beyond, the rounding of t^2 shows
// (8e-6 at -13, where fp32 underflows).  Past 16 nothing is left of Phi(-t).  No branch, 13 operations in pairs, and two results
// of the special-function unit.
template <int N> __device__ __forceinline__ void gelu(float *f)
{
    constexpr float kE[8] = {0.0356747806f, -0.157203093f, 0.206353486f, -0.0536836348f, 0.128561616f, 0.0999135002f, 0.120753959f, 0.119629301f};
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const float z0 = f[i], z1 = f[i + (N > 1)];
        const float2 t = make_float2(fminf(fabsf(z0), 16.f), fminf(fabsf(z1), 16.f));
        const float2 d = fma2(t, both(0.3f), both(1.f)), s = make_float2(rcp(d.x), rcp(d.y));
        float2 e = both(kE[0]);
#pragma unroll
        for (int k = 1; k < 8; ++k) e = fma2(e, s, both(kE[k]));
        const float2 power = mul2(mul2(t, t), both(-0.5f * kLog2e));
        const float2 q = mul2(mul2(e, s), make_float2(ex2(power.x), ex2(power.y)));
        const float2 r = fma2(make_float2(-t.x, -t.y), q, make_float2(max_nan(z0, 0.f), max_nan(z1, 0.f)));
        f[i] = r.x;
        if (N > 1) f[i + 1] = r.y;
    }
}

template <int ACT, int N> __device__ __forceinline__ void activate(float *f)
{
    if constexpr (ACT == SPDY_ACT_GELU) {
        gelu<N>(f);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (ACT == SPDY_ACT_RELU) f[i] = max_nan(f[i], 0.f);
            if (ACT == SPDY_ACT_SILU) f[i] = f[i] == neg_inf() ? 0.f : __fdividef(f[i], 1.f + ex2(-f[i] * kLog2e));
        }
    }
}

__device__ __forceinline__ float bias_at(const LinearArgs &a, int64_t n)
{
    if (a.bias_type == SPDY_F32) return static_cast<const float *>(a.bias)[n];
    if (a.bias_type == SPDY_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(a.bias)[n]);
    return __half2float(static_cast<const __half *>(a.bias)[n]);
}

// bias[n .. n+7], 0 beyond N
template <class T> __device__ __forceinline__ void bias8(const LinearArgs &a, int64_t n, float *b)
{
    if (a.bias && a.wide_bias && n + 8 <= a.N) {
        if (a.bias_type == SPDY_F32) {
            Elem<float>::unpack(reinterpret_cast<const uint4 *>(static_cast<const float *>(a.bias) + n)[0], b);
            Elem<float>::unpack(reinterpret_cast<const uint4 *>(static_cast<const float *>(a.bias) + n)[1], b + 4);
        } else {
            Elem<T>::unpack(*reinterpret_cast<const uint4 *>(static_cast<const T *>(a.bias) + n), b);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = a.bias && n + i < a.N ? bias_at(a, n + i) : 0.f;
}

// residual[m][n .. n+7] as they lie, 0 beyond the matrix
template <class T> __device__ __forceinline__ uint4 residual8(const LinearArgs &a, int64_t m, int64_t n)
{
    if (!a.residual || m >= a.M || n >= a.N) return make_uint4(0, 0, 0, 0);
    const T *p = static_cast<const T *>(a.residual) + m * a.ldres + n;
    if (a.wide_res && n + 8 <= a.N) return *reinterpret_cast<const uint4 *>(p);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = n + i < a.N ? Elem<T>::to_float(p[i]) : 0.f;
    return Elem<T>::pack(f);
}

// Stores elements n .. n+7 of row m.
template <class T> __device__ __forceinline__ void store8(const LinearArgs &a, int64_t m, int64_t n, const float *f)
{
    if (m >= a.M || n >= a.N) return;
    const bool whole = n + 8 <= a.N && a.wide_out;
    if (a.out_type == SPDY_F32) {
        float *q = static_cast<float *>(a.y) + m * a.ldy + n;
        if (whole) {
            reinterpret_cast<float4 *>(q)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4 *>(q)[1] = make_float4(f[4], f[5], f[6], f[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (n + i < a.N) q[i] = f[i];
        }
        return;
    }
    T *q = static_cast<T *>(a.y) + m * a.ldy + n;
    if (whole) {
        *reinterpret_cast<uint4 *>(q) = Elem<T>::pack(f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n + i < a.N) q[i] = Elem<T>::from_float(f[i]);
    }
}

// Activation and residual of eight sums, bias included.
template <class T, int ACT> __device__ __forceinline__ void finish8(const LinearArgs &a, float *f, uint4 residual)
{
    activate<ACT, 8>(f);
    if (a.residual) {
        float res[8];
        Elem<T>::unpack(residual, res);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += res[i];
    }
}

// 16 columns (from n) of 32 rows (from m), a row to a lane, stored by runs of columns; 1 KB of shared memory of the warp's own.
// The values come by value: an address would put them into local memory on the fast way too.
__device__ __noinline__ void turn_wide(const LinearArgs &a, int64_t m, int64_t n, uint4 v0, uint4 v1, uint4 v2, uint4 v3, unsigned char *turn)
{
    const int lane = threadIdx.x & 31;
    uint4 *mine = reinterpret_cast<uint4 *>(turn);
    for (int half = 0; half < 2; ++half) {
        __syncwarp();
        mine[2 * lane] = half ? v2 : v0;
        mine[2 * lane + 1] = half ? v3 : v1;
        __syncwarp();
#pragma unroll
        for (int it = 0; it < 8; ++it) {
            const int64_t row = m + it * 4 + lane / 8, col = n + half * 8 + lane % 8;
            if (row < a.M && col < a.N) static_cast<float *>(a.y)[row * a.ldy + col] = reinterpret_cast<const float *>(turn)[it * 32 + lane];
        }
    }
}
__device__ __noinline__ void turn_narrow(const LinearArgs &a, int64_t m, int64_t n, uint4 v0, uint4 v1, unsigned char *turn)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
    reinterpret_cast<uint4 *>(turn)[2 * lane] = v0;
    reinterpret_cast<uint4 *>(turn)[2 * lane + 1] = v1;
    __syncwarp();
    uint16_t *y = static_cast<uint16_t *>(a.y);
    if (a.words && n + 16 <= a.N) {  // two columns to a lane
        uint32_t v[8];
#pragma unroll
        for (int it = 0; it < 8; ++it) v[it] = reinterpret_cast<const uint32_t *>(turn)[it * 32 + lane];
#pragma unroll
        for (int it = 0; it < 8; ++it) {
            const int64_t row = m + it * 4 + lane / 8;
            if (row < a.M) *reinterpret_cast<uint32_t *>(y + row * a.ldy + n + lane % 8 * 2) = v[it];
        }
        return;
    }
#pragma unroll
    for (int it = 0; it < 16; ++it) {
        const int64_t row = m + it * 2 + lane / 16, col = n + lane % 16;
        if (row < a.M && col < a.N) y[row * a.ldy + col] = reinterpret_cast<const uint16_t *>(turn)[it * 32 + lane];
    }
}

// NaN in `cols` columns (from n) of a warp's 32 rows (from m): a tile whose products never came.
__device__ __noinline__ void spoil(const LinearArgs &a, int64_t m, int64_t n, int cols)
{
    m += threadIdx.x & 31;
    if (m >= a.M) return;
    for (int c = 0; c < cols && n + c < a.N; ++c) {
        if (a.out_type == SPDY_F32) static_cast<float *>(a.y)[m * a.ldy + n + c] = quiet_nan();
        else static_cast<uint16_t *>(a.y)[m * a.ldy + n + c] = 0x7fffu;  // in bf16 and in f16
    }
}

// One warp carries COLS columns of its 32 rows (from row m0) of an accumulator at `tmem` to y, 16 columns at a time: a lane holds
// a row, 16 columns of it, and touches y and residual in whole 32-byte sectors.  (Turning the rows through shared memory for
// longer runs cost more than it gave: the tensor core's operands and the copies that bring them take the shared memory's
// bandwidth.)  `bias` is the warp's own COLS floats of shared memory.  The next 16 columns' residual is fetched before the
// present ones are worked on, the first before the accumulator is waited for (`ready`); `release` is called once the last
// columns have left TMEM.  Rows that start anywhere go through 1 KB of shared memory (`turn`), so that a store covers runs of
// columns rather than single elements of 32 rows.
// FAST: all columns lie inside and every row starts on 32 bytes.
template <class T, int ACT, int COLS, bool RES, bool FAST, class Ready, class Release>
__device__ __forceinline__ void carry(const LinearArgs &a, uint32_t tmem, int64_t m0, int64_t n0, float *bias, unsigned char *turn, Ready ready, Release release)
{
    const int lane = threadIdx.x & 31;
    const int64_t m = m0 + lane;
    const bool inside = m < a.M;
    const T *from = RES ? static_cast<const T *>(a.residual) + m * a.ldres + n0 : nullptr;
    char *to = static_cast<char *>(a.y) + (m * a.ldy + n0) * (a.out_type == SPDY_F32 ? 4 : 2);
    uint4 next[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    const auto fetch = [&](int c) {
        if (!RES) return;
        if (FAST) {
            if (inside) load32(from + c, next[0], next[1]);
        } else {
            next[0] = residual8<T>(a, m, n0 + c), next[1] = residual8<T>(a, m, n0 + c + 8);
        }
    };
    __syncwarp();
    for (int i = lane; i < COLS; i += 32) bias[i] = a.bias && n0 + i < a.N ? bias_at(a, n0 + i) : 0.f;
    fetch(0);
    __syncwarp();
    if (!ready()) return spoil(a, m0, n0, COLS);
#pragma unroll 1
    for (int c = 0; c < COLS; c += 16) {
        float f[16];
        tmem_load16(tmem + c, f);
        if (c + 16 == COLS) release();
        const uint4 res[2] = {next[0], next[1]};
        if (c + 16 < COLS) fetch(c + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 b = reinterpret_cast<const float4 *>(bias + c)[i];
            f[4 * i] += b.x, f[4 * i + 1] += b.y, f[4 * i + 2] += b.z, f[4 * i + 3] += b.w;
        }
        activate<ACT, 16>(f);
        if (RES) {
            float r[16];
            Elem<T>::unpack(res[0], r), Elem<T>::unpack(res[1], r + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] += r[i];
        }
        if (!FAST) {
            if (a.out_type == SPDY_F32) turn_wide(a, m0, n0 + c, Elem<float>::pack(f), Elem<float>::pack(f + 4), Elem<float>::pack(f + 8), Elem<float>::pack(f + 12), turn);
            else turn_narrow(a, m0, n0 + c, Elem<T>::pack(f), Elem<T>::pack(f + 8), turn);
        } else if (inside) {
            if (a.out_type == SPDY_F32) {
                store32(to + 4 * c, Elem<float>::pack(f), Elem<float>::pack(f + 4));
                store32(to + 4 * c + 32, Elem<float>::pack(f + 8), Elem<float>::pack(f + 12));
            } else {
                store32(to + 2 * c, Elem<T>::pack(f), Elem<T>::pack(f + 8));
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- tensor-core kernel
enum { kAlone = 0, kSplit = 1, kPair = 2 };

template <int BN, int MODE> struct Shape {
    static constexpr int kRowsB = MODE == kPair ? BN / 2 : BN;  // rows of w a block holds
    static constexpr int kSliceBytes = (BM + kRowsB) * BK * 2;  // x's rows, then w's
    static constexpr int kStageBytes = kSlices * kSliceBytes;
    static constexpr int kStages = 196608 / kStageBytes;
    static constexpr int kTmemColumns = 2 * BN;
    // behind the stages: the parts of a tile (kSplit), or the epilogue warps' bias and room to turn rows
    static constexpr int kWarpColumns = BN / 4 < 32 ? 32 : BN / 4;  // of an epilogue warp; the warps beyond BN have none
    static constexpr int kWorkers = 4 * (BN / kWarpColumns);
    static constexpr int kExtra = MODE == kSplit ? BM * BN * 4 : kWorkers * (kWarpColumns * 4 + 1024);
    static constexpr int kSmem = 1024 + kStages * kStageBytes + kExtra;
};

struct Control {
    uint64_t full[8], empty[8], acc_full[2], acc_empty[2];
    uint32_t tmem;
};

// Two accumulators in TMEM, so that a tile's epilogue runs beside the next tile's products.
//   kAlone: persistent blocks walk over tiles of 128 rows.
//   kPair:  persistent pairs of blocks walk over tiles of 256 rows; each block brings its 128 rows of x and half of the tile's rows
//           of w, the first block issues the products of both, each block's TMEM receives its own rows.
//   kSplit (few tiles): a cluster of blocks shares one tile of 128 rows, each multiplying a part of K; the parts meet in the
//           shared memory of the block that owns the columns, and are added there in the order of the blocks.
template <class T, int BN, int ACT, int MODE>
__global__ void __launch_bounds__(kThreads, 1) linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const LinearArgs a)
{
    using S = Shape<BN, MODE>;
    extern __shared__ unsigned char raw_smem[];
    unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *extra = stages + S::kStages * S::kStageBytes;
    __shared__ Control ctl;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = MODE == kAlone ? 1 : static_cast<int>(cluster.num_blocks()), part = MODE == kAlone ? 0 : static_cast<int>(cluster.block_rank());
    const int tiles = a.tiles_m * a.tiles_n;
    const int first = static_cast<int>(blockIdx.x) / parts, step = MODE == kSplit ? tiles : static_cast<int>(gridDim.x) / parts;
    const int kb0 = MODE == kSplit ? static_cast<int>(static_cast<int64_t>(a.k_blocks) * part / parts) : 0;
    const int kb1 = MODE == kSplit ? static_cast<int>(static_cast<int64_t>(a.k_blocks) * (part + 1) / parts) : a.k_blocks;
    constexpr int TILE_M = MODE == kPair ? 2 * BM : BM;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) barrier_init(&ctl.full[i], 1), barrier_init(&ctl.empty[i], 1);
        for (int i = 0; i < 2; ++i) barrier_init(&ctl.acc_full[i], 1), barrier_init(&ctl.acc_empty[i], (MODE == kPair ? 2 : 1) * S::kWorkers);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_x)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_w)) : "memory");
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<MODE == kPair>(&ctl.tmem, S::kTmemColumns);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (MODE != kAlone) cluster.sync();  // other blocks signal this one's barriers or write its shared memory
    else __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = ctl.tmem;

    if (warp == 0) {
        int stage = 0;
        uint32_t parity = 0;
        bool ok = true;
        int issued = 0;
        for (int tile = first; tile < tiles && ok; tile += step) {
            const int m0 = tile % a.tiles_m * TILE_M + (MODE == kPair ? part * BM : 0), n0 = tile / a.tiles_m * BN + (MODE == kPair ? part * S::kRowsB : 0);
            for (int kb = kb0; kb < kb1; ++kb) {
                ok = __all_sync(0xffffffffu, barrier_wait(&ctl.empty[stage], parity ^ 1));
                if (!ok) break;
                unsigned char *to = stages + stage * S::kStageBytes;
                if (elect()) {
                    if (MODE == kPair) {  // both blocks' copies count on the first block's barrier
                        const uint32_t full = first_blocks(smem_addr(&ctl.full[stage]));
                        if (part == 0) barrier_expect(&ctl.full[stage], 2 * S::kStageBytes);
#pragma unroll
                        for (int q = 0; q < kSlices; ++q) {
                            tma_load_pair(to + q * S::kSliceBytes, &map_x, (kb * kSlices + q) * BK, m0, full);
                            tma_load_pair(to + q * S::kSliceBytes + BM * BK * 2, &map_w, (kb * kSlices + q) * BK, n0, full);
                        }
                    } else {
                        barrier_expect(&ctl.full[stage], S::kStageBytes);
#pragma unroll
                        for (int q = 0; q < kSlices; ++q) {
                            tma_load(to + q * S::kSliceBytes, &map_x, (kb * kSlices + q) * BK, m0, &ctl.full[stage]);
                            tma_load(to + q * S::kSliceBytes + BM * BK * 2, &map_w, (kb * kSlices + q) * BK, n0, &ctl.full[stage]);
                        }
                    }
                }
                __syncwarp();
                ++issued;
                if (++stage == S::kStages) stage = 0, parity ^= 1;
            }
        }
        // no copy outlives the block, whatever the other warps met (of a pair, both blocks' are counted on the first one's barriers)
        if (MODE != kPair || part == 0)
            for (int i = 0; i < S::kStages && i < issued; ++i) {
                const int n = issued - 1 - i;
                barrier_wait(&ctl.full[n % S::kStages], n / S::kStages & 1);
            }
    } else if (warp == 1) {
        if (MODE != kPair || part == 0) {
            constexpr uint32_t format = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            constexpr uint32_t idesc = 1u << 4 | format << 7 | format << 10 | static_cast<uint32_t>(BN / 8) << 17 | static_cast<uint32_t>(TILE_M / 16) << 24;
            int stage = 0, acc = 0, issued = 0;
            uint32_t parity = 0, acc_parity = 0;
            bool ok = true;
            for (int tile = first; tile < tiles && ok; tile += step) {
                ok = __all_sync(0xffffffffu, barrier_wait(&ctl.acc_empty[acc], acc_parity ^ 1));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d = tmem + acc * BN;
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = __all_sync(0xffffffffu, barrier_wait(&ctl.full[stage], parity));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = smem_addr(stages + stage * S::kStageBytes);
                    if (elect()) {
#pragma unroll
                        for (int q = 0; q < kSlices; ++q) {
                            const uint64_t da = operand(at + q * S::kSliceBytes), db = operand(at + q * S::kSliceBytes + BM * BK * 2);
#pragma unroll
                            for (int k = 0; k < BK / 16; ++k) mma<MODE == kPair>(d, da + 2 * k, db + 2 * k, idesc, kb > kb0 || q > 0 || k > 0);
                        }
                        mma_commit<MODE == kPair>(&ctl.empty[stage]);
                        if (kb + 1 == kb1) mma_commit<MODE == kPair>(&ctl.acc_full[acc]);
                    }
                    __syncwarp();
                    ++issued;
                    if (++stage == S::kStages) stage = 0, parity ^= 1;
                }
                if (++acc == 2) acc = 0, acc_parity ^= 1;
            }
            // nor does a product: TMEM is freed once the last one issued is done
            if (issued > 0) barrier_wait(&ctl.empty[(issued - 1) % S::kStages], (issued - 1) / S::kStages & 1);
        }
    } else if (MODE != kSplit) {
        // warps 4 to 19: a warp reaches the quarter of TMEM's rows that its number names modulo four
        const int quarter = warp & 3, group = (warp - 2) >> 2;
        unsigned char *turn = extra + (warp - 2) * 1024;
        float *bias = reinterpret_cast<float *>(extra + S::kWorkers * 1024) + (warp - 2) * S::kWarpColumns;
        int acc = 0;
        uint32_t acc_parity = 0;
        bool ok = true;
        for (int tile = group * S::kWarpColumns < BN ? first : tiles; tile < tiles; tile += step) {
            const int64_t m0 = static_cast<int64_t>(tile % a.tiles_m) * TILE_M + (MODE == kPair ? part * BM : 0) + quarter * 32;
            const int64_t n0 = static_cast<int64_t>(tile / a.tiles_m) * BN + group * S::kWarpColumns;
            if (!ok) {
                spoil(a, m0, n0, S::kWarpColumns);
                continue;
            }
            const auto ready = [&] {
                ok = __all_sync(0xffffffffu, barrier_wait(&ctl.acc_full[acc], acc_parity));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                return ok;
            };
            const auto release = [&] {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if (MODE == kPair) barrier_arrive_at(first_blocks(smem_addr(&ctl.acc_empty[acc])));
                    else barrier_arrive(&ctl.acc_empty[acc]);
                }
            };
            const uint32_t at = tmem + acc * BN + group * S::kWarpColumns + (static_cast<uint32_t>(quarter * 32) << 16);
            if (a.sectors && n0 + S::kWarpColumns <= a.N) {
                if (a.residual) carry<T, ACT, S::kWarpColumns, true, true>(a, at, m0, n0, bias, turn, ready, release);
                else carry<T, ACT, S::kWarpColumns, false, true>(a, at, m0, n0, bias, turn, ready, release);
            } else {
                if (a.residual) carry<T, ACT, S::kWarpColumns, true, false>(a, at, m0, n0, bias, turn, ready, release);
                else carry<T, ACT, S::kWarpColumns, false, false>(a, at, m0, n0, bias, turn, ready, release);
            }
            if (++acc == 2) acc = 0, acc_parity ^= 1;
        }
    }
    __syncwarp();
    if (MODE == kSplit) {
        const int slice = BN / parts;  // columns this block finishes
        const int quarter = warp & 3, group = (warp - 2) >> 2;
        if (warp >= 2 && group * 16 < BN) {
            const bool ok = __all_sync(0xffffffffu, barrier_wait(&ctl.acc_full[0], 0));
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            for (int c = group * 16; c < BN; c += kEpilogueWarps / 4 * 16) {
                float v[16];
                tmem_load16(tmem + c + (static_cast<uint32_t>(quarter * 32) << 16), v);
                if (!ok)
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = quiet_nan();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int col = c + 4 * i, owner = col / slice;
                    // [part][column group of 4][row] float4: consecutive lanes write consecutive 16 bytes
                    float4 *to = cluster.map_shared_rank(reinterpret_cast<float4 *>(extra), owner) + (part * (slice / 4) + col % slice / 4) * BM + quarter * 32 + lane;
                    *to = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        }
        __syncwarp();
        const int64_t m0 = static_cast<int64_t>(first % a.tiles_m) * BM, n0 = static_cast<int64_t>(first / a.tiles_m) * BN + part * slice;
        const float4 *sums = reinterpret_cast<const float4 *>(extra);
        const int items = static_cast<int>(min(static_cast<int64_t>(BM), a.M - m0)) * (slice / 8);
        // the first round's bias and residual come while the parts are exchanged
        float b[8];
        uint4 res = make_uint4(0, 0, 0, 0);
        const auto place = [&](int i, int64_t &m, int64_t &n, int &row, int &g) { row = i / (slice / 8), g = i % (slice / 8), m = m0 + row, n = n0 + g * 8; };
        int64_t m, n;
        int row, g;
        place(static_cast<int>(threadIdx.x), m, n, row, g);
        if (static_cast<int>(threadIdx.x) < items) bias8<T>(a, n, b), res = residual8<T>(a, m, n);
        cluster.sync();
        for (int i = threadIdx.x; i < items; i += kThreads) {
            if (i >= kThreads) {
                place(i, m, n, row, g);
                bias8<T>(a, n, b), res = residual8<T>(a, m, n);
            }
            float f[8] = {};
            for (int p = 0; p < parts; ++p) {
                const float4 lo = sums[(p * (slice / 4) + 2 * g) * BM + row], hi = sums[(p * (slice / 4) + 2 * g + 1) * BM + row];
                f[0] += lo.x, f[1] += lo.y, f[2] += lo.z, f[3] += lo.w, f[4] += hi.x, f[5] += hi.y, f[6] += hi.z, f[7] += hi.w;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] += b[j];
            finish8<T, ACT>(a, f, res);
            store8<T>(a, m, n, f);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (MODE == kPair) cluster.sync();  // no block leaves while its barriers are signalled or its operands read
    else __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free<MODE == kPair>(tmem, S::kTmemColumns);
    }
}

// ---------------------------------------------------------------------------------------------- few rows
// A block of four warps per COLS columns of y (rows of w) and ROWS rows of x: w is read once per ROWS rows, each warp a quarter of its
// K at a time, x comes from L1; the warps' sums are added in their order.  Bound by w's bytes and the launch: 1 x 768 x 3072 4.1 us,
// 1 x 4096 x 4096 6.3 us (33.6 MB, 5.3 TB/s; w stays in L2 between such calls).
template <class T, int ROWS, int COLS, int ACT, bool WIDE> __global__ void __launch_bounds__(128) linear_rows_kernel(const LinearArgs a)
{
    __shared__ float part[4][ROWS * COLS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n0 = static_cast<int64_t>(blockIdx.x) * COLS, m0 = static_cast<int64_t>(blockIdx.y) * ROWS;
    float acc[ROWS][COLS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < COLS; ++c) acc[r][c] = 0.f;
    const T *x = static_cast<const T *>(a.x) + m0 * a.ldx, *w = static_cast<const T *>(a.w) + n0 * a.ldw;
    if (WIDE) {
#pragma unroll 2
        for (int64_t k = threadIdx.x * 8; k < a.K; k += 1024) {
            uint4 wr[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) wr[c] = n0 + c < a.N ? load_stream(w + c * a.ldw + k) : make_uint4(0, 0, 0, 0);
            float xf[ROWS][8];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) Elem<T>::unpack(m0 + r < a.M ? *reinterpret_cast<const uint4 *>(x + r * a.ldx + k) : make_uint4(0, 0, 0, 0), xf[r]);
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                float wf[8];
                Elem<T>::unpack(wr[c], wf);
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[r][c] = fmaf(xf[r][i], wf[i], acc[r][c]);
            }
        }
    } else {
#pragma unroll 4
        for (int64_t k = threadIdx.x; k < a.K; k += 128) {
            float wf[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) wf[c] = n0 + c < a.N ? Elem<T>::to_float(w[c * a.ldw + k]) : 0.f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float xf = m0 + r < a.M ? Elem<T>::to_float(x[r * a.ldx + k]) : 0.f;
#pragma unroll
                for (int c = 0; c < COLS; ++c) acc[r][c] = fmaf(xf, wf[c], acc[r][c]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
#pragma unroll
            for (int d = 16; d; d >>= 1) acc[r][c] += __shfl_xor_sync(0xffffffffu, acc[r][c], d);
            if (lane == 0) part[warp][r * COLS + c] = acc[r][c];
        }
    __syncthreads();
    const int i = threadIdx.x;
    const int64_t m = m0 + i / COLS, n = n0 + i % COLS;
    if (i >= ROWS * COLS || m >= a.M || n >= a.N) return;
    float z = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
    if (a.bias) z += bias_at(a, n);
    activate<ACT, 1>(&z);
    if (a.residual) z += Elem<T>::to_float(static_cast<const T *>(a.residual)[m * a.ldres + n]);
    if (a.out_type == SPDY_F32) static_cast<float *>(a.y)[m * a.ldy + n] = z;
    else static_cast<T *>(a.y)[m * a.ldy + n] = Elem<T>::from_float(z);
}

// ---------------------------------------------------------------------------------------------- launches
bool on_tensor_cores(int64_t M, int64_t K) { return M > kFewRows && K > 0; }
template <class T, int BN, int ACT, int MODE> int launch_tiles(const CUtensorMap &mx, const CUtensorMap &mw, const LinearArgs &a, int parts, cudaStream_t s)
{
    constexpr int smem = Shape<BN, MODE>::kSmem;
    const int tiles = a.tiles_m * a.tiles_n, units = sm_count() / parts;
    auto *kernel = linear_kernel<T, BN, ACT, MODE>;
    SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>((MODE == kSplit || tiles < units ? tiles : units) * parts));
    config.blockDim = dim3(kThreads);
    config.dynamicSmemBytes = smem;
    config.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(parts);
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    config.attrs = attr;
    config.numAttrs = parts > 1 ? 1 : 0;
    SPDY_EVAL_TRY(cudaLaunchKernelEx(&config, kernel, mx, mw, a));
    return SPDY_OK;
}

// How many clusters of `parts` blocks of the split kernel the device holds at once (a block takes a whole multiprocessor, and a
// cluster lies within one group of them, so that fewer fit than the division says).  Asked once per device and size.
template <class T, int ACT> int split_clusters(int parts)
{
    static int held[64][4];
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess || device < 0 || device >= 64) return 0;
    const int at = parts == 2 ? 1 : parts == 4 ? 2 : 3;
    int n = __atomic_load_n(&held[device][at], __ATOMIC_RELAXED);
    if (n == 0) {
        constexpr int smem = Shape<64, kSplit>::kSmem;
        auto *kernel = linear_kernel<T, 64, ACT, kSplit>;
        cudaLaunchConfig_t config = {};
        config.gridDim = dim3(static_cast<unsigned>(parts * sm_count()));
        config.blockDim = dim3(kThreads);
        config.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = static_cast<unsigned>(parts);
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        config.attrs = attr;
        config.numAttrs = 1;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, kernel, &config) != cudaSuccess || n < 1) {
            (void)cudaGetLastError();
            n = 1;
        }
        __atomic_store_n(&held[device][at], n, __ATOMIC_RELAXED);
    }
    return n;
}

// Which tiles carry a product: the shape with the least estimated time, in cycles per multiprocessor.  A round of tiles costs its
// stages (4096 multiply-adds a cycle at best; a stage's barriers and copies have a floor near 500: measured) and an epilogue that no product hides
// (the last round's).
struct TilePlan {
    int mode, width, parts;
};
template <class T, int ACT> TilePlan choose_tiles(int64_t M, int64_t N, int64_t k_blocks, int sms)
{
    const auto div = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
    struct Option {
        int mode, width, rows, units;
        double per_slice, fixed;
    };
    const Option options[3] = {{kPair, 256, 256, sms / 2, 1040, 4000}, {kAlone, 128, 128, sms, 620, 2500}, {kAlone, 64, 128, sms, 540, 2000}};
    TilePlan best = {kAlone, 64, 1};
    double least = 1e300;
    for (const Option &o : options) {
        const double time = static_cast<double>(div(div(M, o.rows) * div(N, o.width), o.units)) * o.per_slice * static_cast<double>(k_blocks) + o.fixed;
        if (time < least) least = time, best = {o.mode, o.width, o.mode == kPair ? 2 : 1};
    }
    // Tiles that leave most multiprocessors idle share their K among up to 8 of them.
    const int64_t tiles = div(M, 128) * div(N, 64);
    int parts = 1;
    while (parts < 8 && tiles * parts * 2 <= sms && k_blocks >= parts * 2 && tiles <= split_clusters<T, ACT>(parts * 2)) parts *= 2;
    if (parts > 1) best = {kSplit, 64, parts};
    return best;
}

template <class T, int ACT> int launch_product(LinearArgs a, void *workspace, cudaStream_t s)
{
    Repack p = {};
    p.K = a.K, p.ldto = packed_ld(a.K);
    char *ws = static_cast<char *>(workspace);
    if (!tma_ok(a.x, a.ldx)) {
        p.from[0] = static_cast<const uint16_t *>(a.x), p.ld[0] = a.ldx, p.rows[0] = a.M, p.to[0] = reinterpret_cast<uint16_t *>(ws);
        a.x = ws, a.ldx = p.ldto, ws += packed_bytes(a.M, a.K);
    }
    if (!tma_ok(a.w, a.ldw)) {
        p.from[1] = static_cast<const uint16_t *>(a.w), p.ld[1] = a.ldw, p.rows[1] = a.N, p.to[1] = reinterpret_cast<uint16_t *>(ws);
        a.w = ws, a.ldw = p.ldto;
    }
    int rc = repack(p, s);
    if (rc != SPDY_OK) return rc;
    a.k_blocks = static_cast<int>((a.K + BK * kSlices - 1) / (BK * kSlices));
    const TilePlan plan = choose_tiles<T, ACT>(a.M, a.N, a.k_blocks, sm_count());
    const int64_t rows = plan.mode == kPair ? 2 * BM : BM, tm = (a.M + rows - 1) / rows, tn = (a.N + plan.width - 1) / plan.width;
    if (tm * tn > 0x7fffffff / 8) return SPDY_ERR_UNSUPPORTED;
    a.tiles_m = static_cast<int>(tm), a.tiles_n = static_cast<int>(tn);
    CUtensorMap mx, mw;
    rc = make_map(&mx, a.x, a.ldx, a.M, a.K, a.dtype, BM);
    if (rc == SPDY_OK) rc = make_map(&mw, a.w, a.ldw, a.N, a.K, a.dtype, plan.mode == kPair ? plan.width / 2 : plan.width);
    if (rc != SPDY_OK) return rc;
    if (plan.mode == kSplit) return launch_tiles<T, 64, ACT, kSplit>(mx, mw, a, plan.parts, s);
    if (plan.mode == kPair) return launch_tiles<T, 256, ACT, kPair>(mx, mw, a, 2, s);
    return plan.width == 128 ? launch_tiles<T, 128, ACT, kAlone>(mx, mw, a, 1, s) : launch_tiles<T, 64, ACT, kAlone>(mx, mw, a, 1, s);
}

template <class T, int ROWS, int ACT> int launch_rows_of(const LinearArgs &a, cudaStream_t s)
{
    constexpr int COLS = 4;
    const dim3 grid(static_cast<unsigned>((a.N + COLS - 1) / COLS), static_cast<unsigned>((a.M + ROWS - 1) / ROWS));
    if (tma_ok(a.x, a.ldx) && tma_ok(a.w, a.ldw) && a.K % 8 == 0) linear_rows_kernel<T, ROWS, COLS, ACT, true><<<grid, 128, 0, s>>>(a);
    else linear_rows_kernel<T, ROWS, COLS, ACT, false><<<grid, 128, 0, s>>>(a);
    return finish_launch();
}

template <class T, int ACT> int launch_rows(const LinearArgs &a, cudaStream_t s)
{
    if (a.M == 1) return launch_rows_of<T, 1, ACT>(a, s);
    if (a.M == 2) return launch_rows_of<T, 2, ACT>(a, s);
    // A grid's second dimension ends at 65535: rows without products (K = 0) may be more.
    constexpr int64_t most = 65535 * 4;
    LinearArgs some = a;
    for (int64_t m = 0; m < a.M; m += most) {
        some.M = a.M - m < most ? a.M - m : most;
        some.y = static_cast<char *>(a.y) + m * a.ldy * static_cast<int64_t>(type_size(a.out_type));
        if (a.residual) some.residual = static_cast<const T *>(a.residual) + m * a.ldres;
        const int rc = launch_rows_of<T, 4, ACT>(some, s);
        if (rc != SPDY_OK) return rc;
    }
    return SPDY_OK;
}

template <class T, int ACT> int launch(const LinearArgs &a, void *workspace, cudaStream_t s)
{
    return on_tensor_cores(a.M, a.K) ? launch_product<T, ACT>(a, workspace, s) : launch_rows<T, ACT>(a, s);
}

template <class T> int launch_type(const LinearArgs &a, void *workspace, cudaStream_t s)
{
    switch (a.activation) {
        case SPDY_ACT_RELU: return launch<T, SPDY_ACT_RELU>(a, workspace, s);
        case SPDY_ACT_GELU: return launch<T, SPDY_ACT_GELU>(a, workspace, s);
        case SPDY_ACT_SILU: return launch<T, SPDY_ACT_SILU>(a, workspace, s);
        default: return launch<T, SPDY_ACT_NONE>(a, workspace, s);
    }
}

}  // namespace

extern "C" {

size_t spdy_linear_workspace_bytes(const void *x, int64_t ldx, const void *w, int64_t ldw, int dtype, int64_t M, int64_t N, int64_t K)
{
    if (!half_type(dtype) || M <= 0 || N <= 0 || K <= 0 || !on_tensor_cores(M, K)) return 0;
    return (tma_ok(x, ldx) ? 0 : packed_bytes(M, K)) + (tma_ok(w, ldw) ? 0 : packed_bytes(N, K));
}

int spdy_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, int dtype, const void *bias, int bias_dtype, const void *residual, int64_t ldres,
                int activation, int64_t M, int64_t N, int64_t K, void *y, int64_t ldy, int out_dtype, void *workspace, size_t workspace_bytes,
                void *cuda_stream)
{
    constexpr int64_t most = 0x7fffff00;
    if (!half_type(dtype) || !(out_dtype == dtype || out_dtype == SPDY_F32) || activation < SPDY_ACT_NONE || activation > SPDY_ACT_SILU) return SPDY_ERR_INVALID_ARG;
    if (M < 0 || N < 0 || K < 0 || M > most || N > most || K > most || ldx < K || ldw < K || ldy < N || (residual && ldres < N)) return SPDY_ERR_INVALID_ARG;
    if (bias && !(bias_dtype == dtype || bias_dtype == SPDY_F32)) return SPDY_ERR_INVALID_ARG;
    if (M == 0 || N == 0) return SPDY_OK;
    if ((K > 0 && (!x || !w)) || !y || !aligned(x, 2) || !aligned(w, 2) || !aligned(y, type_size(out_dtype)) || !aligned(residual, 2) ||
        (bias && !aligned(bias, type_size(bias_dtype))))
        return SPDY_ERR_INVALID_ARG;
    const size_t need = spdy_linear_workspace_bytes(x, ldx, w, ldw, dtype, M, N, K);
    if (need && (!workspace || !aligned(workspace, 256))) return SPDY_ERR_INVALID_ARG;
    if (workspace_bytes < need) return SPDY_ERR_WORKSPACE_TOO_SMALL;
    LinearArgs a = {};
    a.x = x, a.w = w, a.bias = bias, a.residual = residual, a.y = y;
    a.ldx = ldx, a.ldw = ldw, a.ldres = ldres, a.ldy = ldy, a.M = M, a.N = N, a.K = K;
    a.dtype = dtype, a.bias_type = bias_dtype, a.out_type = out_dtype, a.activation = activation;
    a.wide_out = aligned(y, 16) && ldy * static_cast<int64_t>(type_size(out_dtype)) % 16 == 0;
    a.wide_res = residual && aligned(residual, 16) && ldres % 8 == 0;
    a.wide_bias = aligned(bias, 16);
    a.words = aligned(y, 4) && ldy % 2 == 0;
    a.sectors = aligned(y, 32) && ldy * static_cast<int64_t>(type_size(out_dtype)) % 32 == 0 && (!residual || (aligned(residual, 32) && ldres % 16 == 0));
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return dtype == SPDY_BF16 ? launch_type<__nv_bfloat16>(a, workspace, s) : launch_type<__half>(a, workspace, s);
}

int spdy_linear_check_status(void *cuda_stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int count = 0, more = 0;
    int rc = take_timeouts(s, &count);
    if (rc == SPDY_OK) rc = linear_logprobs_timeouts(s, &more);
    if (rc != SPDY_OK) return rc;
    return count + more == 0 ? SPDY_OK : SPDY_ERR_INTERNAL;
}

}  // extern "C"
