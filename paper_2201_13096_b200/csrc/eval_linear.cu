// y = act(x w^T + bias) + residual: kernels and C entry (spdy_eval.h).
//
// The product runs on the tensor cores (tcgen05, 16-bit operands, fp32 accumulators in TMEM); one thread feeds it with TMA
// copies of 64-wide slices of x and w, one issues the matrix instructions, eight warps carry the finished tiles through the
// epilogue while the next tile is multiplied.  Few rows (single tokens) are a matter of reading w once: a kernel of plain
// multiply-adds streams it.
#include <cuda.h>

#include "eval_common.cuh"

using namespace spdy_eval;

namespace {

namespace cg = cooperative_groups;

constexpr int BM = 128, BK = 64;           // rows of a tile; depth of a stage: 64 16-bit elements = one 128-byte swizzle row
constexpr int kEpilogueWarps = 8;
constexpr int kThreads = 32 * (2 + kEpilogueWarps);
constexpr int64_t kFewRows = 8;            // at most this many rows take the multiply-add kernel

struct LinearArgs {
    const void *x, *w, *bias, *residual;
    void *y;
    int64_t ldx, ldw, ldres, ldy, M, N, K;
    int dtype, bias_type, out_type, activation;
    int tiles_m, tiles_n, k_blocks;
    int wide_out, wide_res;                // 16-byte accesses are possible on every row of y, of residual
};

__device__ int g_timeouts;                 // waits that ran out of time (none in a working run); spdy_linear_check_status

// ---------------------------------------------------------------------------------------------- mbarrier, TMA, tcgen05
__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void barrier_init(uint64_t *b, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count) : "memory"); }
__device__ __forceinline__ void barrier_arrive(uint64_t *b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory"); }
__device__ __forceinline__ void barrier_expect(uint64_t *b, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(b)), "r"(bytes) : "memory");
}
// Waits until the phase of `parity` is over; gives up after about two seconds and counts that.
__device__ __forceinline__ bool barrier_wait(uint64_t *b, uint32_t parity)
{
    const uint32_t addr = smem_addr(b);
    long long start = 0;
    for (;;) {
        uint32_t done;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(done)
            : "r"(addr), "r"(parity)
            : "memory");
        if (done) return true;
        const long long now = clock64();
        if (start == 0) start = now;
        if (now - start > 4000000000ll) {
            atomicAdd(&g_timeouts, 1);
            return false;
        }
    }
}
__device__ __forceinline__ void tma_load(void *to, const CUtensorMap *map, int x, int y, uint64_t *b)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_addr(to)),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_addr(b))
                 : "memory");
}
// Descriptor of a K-major operand whose rows are 128 bytes under the 128-byte swizzle: groups of 8 rows lie 1024 bytes apart.
__device__ __forceinline__ uint64_t operand(uint32_t addr) { return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | 1ull << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61; }

__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                 "r"(static_cast<uint32_t>(add))
                 : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t *b)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(b)) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t *v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
        "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
          "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]),
          "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr)
        : "memory");
}

// ---------------------------------------------------------------------------------------------- epilogue
template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if (ACT == SPDY_ACT_RELU) return max_nan(z, 0.f);
    if (ACT == SPDY_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
    if (ACT == SPDY_ACT_SILU) return z == neg_inf() ? 0.f : __fdividef(z, 1.f + ex2(-z * kLog2e));
    return z;
}

__device__ __forceinline__ float bias_at(const LinearArgs &a, int64_t n)
{
    if (a.bias_type == SPDY_F32) return static_cast<const float *>(a.bias)[n];
    if (a.bias_type == SPDY_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(a.bias)[n]);
    return __half2float(static_cast<const __half *>(a.bias)[n]);
}

// Activation, residual and the store of elements n .. n+7 of row m, whose sums (bias included) are in f.
template <class T, int ACT> __device__ __forceinline__ void finish8(const LinearArgs &a, int64_t m, int64_t n, float *f)
{
    const bool whole = n + 8 <= a.N;
    float res[8];
    if (a.residual) {
        const T *p = static_cast<const T *>(a.residual) + m * a.ldres + n;
        if (whole && a.wide_res) {
            Elem<T>::unpack(*reinterpret_cast<const uint4 *>(p), res);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) res[i] = n + i < a.N ? Elem<T>::to_float(p[i]) : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f[i] = activate<ACT>(f[i]);
        if (a.residual) f[i] += res[i];
    }
    if (a.out_type == SPDY_F32) {
        float *q = static_cast<float *>(a.y) + m * a.ldy + n;
        if (whole && a.wide_out) {
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
    if (whole && a.wide_out) {
        *reinterpret_cast<uint4 *>(q) = Elem<T>::pack(f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (n + i < a.N) q[i] = Elem<T>::from_float(f[i]);
    }
}

// ---------------------------------------------------------------------------------------------- tensor-core kernel
template <int BN> struct Shape {
    static constexpr int kStageBytes = (BM + BN) * BK * 2;
    static constexpr int kStages = BN == 256 ? 4 : BN == 128 ? 6 : 8;
    static constexpr int kTmemColumns = 2 * BN;
    static constexpr int kSmem = 1024 + kStages * kStageBytes + kEpilogueWarps * 4096 + 256;
};

struct Control {
    uint64_t full[8], empty[8], acc_full[2], acc_empty[2];
    uint32_t tmem;
};

// SPLIT false: persistent blocks walk over the tiles, two accumulators in TMEM so that a tile's epilogue runs beside the next
// tile's products.  SPLIT true (few tiles): a cluster of blocks shares one tile, each multiplying a part of K; the parts
// meet in the shared memory of the block that owns the columns, and are added there in the order of the blocks.
template <class T, int BN, int ACT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1) linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const LinearArgs a)
{
    using S = Shape<BN>;
    extern __shared__ unsigned char raw_smem[];
    unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *staging = stages + S::kStages * S::kStageBytes;
    __shared__ Control ctl;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int parts = SPLIT ? static_cast<int>(cluster.num_blocks()) : 1, part = SPLIT ? static_cast<int>(cluster.block_rank()) : 0;
    const int tiles = a.tiles_m * a.tiles_n;
    const int first = SPLIT ? static_cast<int>(blockIdx.x) / parts : static_cast<int>(blockIdx.x), step = SPLIT ? tiles : static_cast<int>(gridDim.x);
    const int kb0 = static_cast<int>(static_cast<int64_t>(a.k_blocks) * part / parts), kb1 = static_cast<int>(static_cast<int64_t>(a.k_blocks) * (part + 1) / parts);

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) barrier_init(&ctl.full[i], 1), barrier_init(&ctl.empty[i], 1);
        for (int i = 0; i < 2; ++i) barrier_init(&ctl.acc_full[i], 1), barrier_init(&ctl.acc_empty[i], kEpilogueWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl.tmem)), "r"(S::kTmemColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = ctl.tmem;

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0;
            uint32_t parity = 0;
            bool ok = true;
            int issued = 0;
            for (int tile = first; tile < tiles && ok; tile += step) {
                const int m0 = tile % a.tiles_m * BM, n0 = tile / a.tiles_m * BN;
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = barrier_wait(&ctl.empty[stage], parity ^ 1);
                    if (!ok) break;
                    unsigned char *to = stages + stage * S::kStageBytes;
                    barrier_expect(&ctl.full[stage], S::kStageBytes);
                    tma_load(to, &map_x, kb * BK, m0, &ctl.full[stage]);
                    tma_load(to + BM * BK * 2, &map_w, kb * BK, n0, &ctl.full[stage]);
                    ++issued;
                    if (++stage == S::kStages) stage = 0, parity ^= 1;
                }
            }
            if (!ok)  // copies in flight may not outlive the block
                for (int i = 0; i < S::kStages && i < issued; ++i) {
                    const int n = issued - 1 - i;
                    barrier_wait(&ctl.full[n % S::kStages], n / S::kStages & 1);
                }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            constexpr uint32_t format = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            constexpr uint32_t idesc = 1u << 4 | format << 7 | format << 10 | static_cast<uint32_t>(BN / 8) << 17 | static_cast<uint32_t>(BM / 16) << 24;
            int stage = 0, acc = 0;
            uint32_t parity = 0, acc_parity = 0;
            bool ok = true;
            for (int tile = first; tile < tiles && ok; tile += step) {
                ok = barrier_wait(&ctl.acc_empty[acc], acc_parity ^ 1);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t d = tmem + acc * BN;
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = barrier_wait(&ctl.full[stage], parity);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = smem_addr(stages + stage * S::kStageBytes);
                    const uint64_t da = operand(at), db = operand(at + BM * BK * 2);
#pragma unroll
                    for (int k = 0; k < BK / 16; ++k) mma(d, da + 2 * k, db + 2 * k, idesc, kb > kb0 || k > 0);
                    mma_commit(&ctl.empty[stage]);
                    if (++stage == S::kStages) stage = 0, parity ^= 1;
                }
                if (!ok) break;
                mma_commit(&ctl.acc_full[acc]);
                if (++acc == 2) acc = 0, acc_parity ^= 1;
            }
        }
    } else if (!SPLIT) {
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        float4 *mine = reinterpret_cast<float4 *>(staging + (warp - 2) * 4096);
        int acc = 0;
        uint32_t acc_parity = 0;
        for (int tile = first; tile < tiles; tile += step) {
            if (!barrier_wait(&ctl.acc_full[acc], acc_parity)) break;
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int64_t m0 = static_cast<int64_t>(tile % a.tiles_m) * BM + quarter * 32, n0 = static_cast<int64_t>(tile / a.tiles_m) * BN + half * (BN / 2);
#pragma unroll 1
            for (int c = 0; c < BN / 2; c += 32) {
                uint32_t v[32];
                tmem_load32(tmem + acc * BN + half * (BN / 2) + c + (static_cast<uint32_t>(quarter * 32) << 16), v);
                if (c + 32 == BN / 2) {  // the accumulator is free once its last columns are out
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) barrier_arrive(&ctl.acc_empty[acc]);
                }
                // a lane holds a row of 32 columns; turned so that four lanes hold a row of eight each, for whole sectors
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    mine[lane * 8 + (i ^ (lane & 7))] =
                        make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
                __syncwarp();
                const int64_t n = n0 + c + (lane & 3) * 8;
                float b[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) b[i] = a.bias && n + i < a.N ? bias_at(a, n + i) : 0.f;
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const int row = it * 8 + (lane >> 2);
                    const float4 lo = mine[row * 8 + ((2 * (lane & 3)) ^ (row & 7))], hi = mine[row * 8 + ((2 * (lane & 3) + 1) ^ (row & 7))];
                    float f[8] = {lo.x + b[0], lo.y + b[1], lo.z + b[2], lo.w + b[3], hi.x + b[4], hi.y + b[5], hi.z + b[6], hi.w + b[7]};
                    if (m0 + row < a.M && n < a.N) finish8<T, ACT>(a, m0 + row, n, f);
                }
            }
            if (++acc == 2) acc = 0, acc_parity ^= 1;
        }
    }
    __syncwarp();
    if (SPLIT) {
        const int slice = BN / parts;  // columns this block finishes
        bool ok = true;
        if (warp >= 2) ok = barrier_wait(&ctl.acc_full[0], 0);
        __syncwarp();
        cluster.sync();  // every block's products are done: the stages may be overwritten
        if (warp >= 2 && ok) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int quarter = warp & 3, half = (warp - 2) >> 2;
#pragma unroll 1
            for (int c = half * (BN / 2); c < (half + 1) * (BN / 2); c += 32) {
                uint32_t v[32];
                tmem_load32(tmem + c + (static_cast<uint32_t>(quarter * 32) << 16), v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int col = c + 4 * i, owner = col / slice;
                    // [part][column group of 4][row] float4: consecutive lanes write consecutive 16 bytes
                    float4 *to = cluster.map_shared_rank(reinterpret_cast<float4 *>(stages), owner) + (part * (slice / 4) + col % slice / 4) * BM + quarter * 32 + lane;
                    *to = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        }
        cluster.sync();
        const int64_t m0 = static_cast<int64_t>(first % a.tiles_m) * BM, n0 = static_cast<int64_t>(first / a.tiles_m) * BN + part * slice;
        const float4 *sums = reinterpret_cast<const float4 *>(stages);
        for (int i = threadIdx.x; i < BM * (slice / 8); i += kThreads) {
            const int row = i / (slice / 8), g = i % (slice / 8);
            const int64_t n = n0 + g * 8;
            if (m0 + row >= a.M || n >= a.N) continue;
            float f[8] = {};
            for (int p = 0; p < parts; ++p) {
                const float4 lo = sums[(p * (slice / 4) + 2 * g) * BM + row], hi = sums[(p * (slice / 4) + 2 * g + 1) * BM + row];
                f[0] += lo.x, f[1] += lo.y, f[2] += lo.z, f[3] += lo.w, f[4] += hi.x, f[5] += hi.y, f[6] += hi.z, f[7] += hi.w;
            }
            if (a.bias)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (n + j < a.N) f[j] += bias_at(a, n + j);
            finish8<T, ACT>(a, m0 + row, n, f);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kTmemColumns) : "memory");
    }
}

// ---------------------------------------------------------------------------------------------- few rows
// One warp per COLS columns of y (rows of w) and ROWS rows of x: w is read once, x comes from L1.
template <class T, int ROWS, int COLS, int ACT, bool WIDE> __global__ void __launch_bounds__(128) linear_rows_kernel(const LinearArgs a)
{
    const int lane = threadIdx.x & 31;
    const int64_t n0 = (static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5)) * COLS, m0 = static_cast<int64_t>(blockIdx.y) * ROWS;
    if (n0 >= a.N) return;
    float acc[ROWS][COLS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < COLS; ++c) acc[r][c] = 0.f;
    const T *x = static_cast<const T *>(a.x) + m0 * a.ldx, *w = static_cast<const T *>(a.w) + n0 * a.ldw;
    if (WIDE) {
#pragma unroll 2
        for (int64_t k = lane * 8; k < a.K; k += 256) {
            float wf[COLS][8];
#pragma unroll
            for (int c = 0; c < COLS; ++c) Elem<T>::unpack(n0 + c < a.N ? load_stream(w + c * a.ldw + k) : make_uint4(0, 0, 0, 0), wf[c]);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (m0 + r >= a.M) break;
                float xf[8];
                Elem<T>::unpack(*reinterpret_cast<const uint4 *>(x + r * a.ldx + k), xf);
#pragma unroll
                for (int c = 0; c < COLS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[r][c] = fmaf(xf[i], wf[c][i], acc[r][c]);
            }
        }
    } else {
        for (int64_t k = lane; k < a.K; k += 32) {
            float wf[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) wf[c] = n0 + c < a.N ? Elem<T>::to_float(w[c * a.ldw + k]) : 0.f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (m0 + r >= a.M) break;
                const float xf = Elem<T>::to_float(x[r * a.ldx + k]);
#pragma unroll
                for (int c = 0; c < COLS; ++c) acc[r][c] = fmaf(xf, wf[c], acc[r][c]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < COLS; ++c)
#pragma unroll
            for (int d = 16; d; d >>= 1) acc[r][c] += __shfl_xor_sync(0xffffffffu, acc[r][c], d);
    // lane r * COLS + c finishes element (r, c)
    float z = 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int c = 0; c < COLS; ++c)
            if (lane == r * COLS + c) z = acc[r][c];
    const int64_t m = m0 + lane / COLS, n = n0 + lane % COLS;
    if (lane >= ROWS * COLS || m >= a.M || n >= a.N) return;
    if (a.bias) z += bias_at(a, n);
    z = activate<ACT>(z);
    if (a.residual) z += Elem<T>::to_float(static_cast<const T *>(a.residual)[m * a.ldres + n]);
    if (a.out_type == SPDY_F32) static_cast<float *>(a.y)[m * a.ldy + n] = z;
    else static_cast<T *>(a.y)[m * a.ldy + n] = Elem<T>::from_float(z);
}

// Copies of operands whose rows TMA cannot read (a row has to start on 16 bytes), with rows of ldto elements.
struct Repack {
    const uint16_t *from[2];
    uint16_t *to[2];
    int64_t ld[2], rows[2], K, ldto;
};
__global__ void __launch_bounds__(256) repack_kernel(const Repack p)
{
    const int which = blockIdx.y;
    if (!p.to[which]) return;
    for (int64_t r = blockIdx.x; r < p.rows[which]; r += gridDim.x) {
        const uint16_t *from = p.from[which] + r * p.ld[which];
        uint16_t *to = p.to[which] + r * p.ldto;
        for (int64_t k = threadIdx.x; k < p.K; k += 256) to[k] = from[k];
    }
}

// ---------------------------------------------------------------------------------------------- launches
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

int make_map(CUtensorMap *map, const void *p, int64_t ld, int64_t rows, int64_t K, int dtype, int box_rows)
{
    EncodeTiled encode = encode_tiled();
    if (!encode) return SPDY_ERR_UNSUPPORTED;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(K), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(ld) * 2};
    const cuuint32_t box[2] = {BK, static_cast<cuuint32_t>(box_rows)}, steps[2] = {1, 1};
    const CUresult rc = encode(map, dtype == SPDY_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(p), dims, strides, box,
                               steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? SPDY_OK : SPDY_ERR_UNSUPPORTED;
}

bool tma_ok(const void *p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0 && ld * 2 < (1ll << 40); }
bool on_tensor_cores(int64_t M, int64_t K) { return M > kFewRows && K > 0; }
int64_t packed_ld(int64_t K) { return (K + 7) / 8 * 8; }
size_t packed_bytes(int64_t rows, int64_t K) { return (static_cast<size_t>(rows) * static_cast<size_t>(packed_ld(K)) * 2 + 255) / 256 * 256; }

template <class T, int BN, int ACT> int launch_tiles(const CUtensorMap &mx, const CUtensorMap &mw, const LinearArgs &a, int parts, cudaStream_t s)
{
    constexpr int smem = Shape<BN>::kSmem;
    const int tiles = a.tiles_m * a.tiles_n;
    cudaLaunchConfig_t config = {};
    config.blockDim = dim3(kThreads);
    config.dynamicSmemBytes = smem;
    config.stream = s;
    cudaLaunchAttribute attr[1];
    config.attrs = attr;
    if (parts > 1) {
        if constexpr (BN <= 64) {
            auto *kernel = linear_kernel<T, BN, ACT, true>;
            SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = static_cast<unsigned>(parts);
            attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
            config.numAttrs = 1;
            config.gridDim = dim3(static_cast<unsigned>(tiles * parts));
            SPDY_EVAL_TRY(cudaLaunchKernelEx(&config, kernel, mx, mw, a));
            return SPDY_OK;
        }
    }
    auto *kernel = linear_kernel<T, BN, ACT, false>;
    SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    config.gridDim = dim3(static_cast<unsigned>(tiles < sm_count() ? tiles : sm_count()));
    SPDY_EVAL_TRY(cudaLaunchKernelEx(&config, kernel, mx, mw, a));
    return SPDY_OK;
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
    if (p.to[0] || p.to[1]) {
        const int64_t rows = p.rows[0] > p.rows[1] ? p.rows[0] : p.rows[1];
        repack_kernel<<<dim3(static_cast<unsigned>(rows < 1184 ? rows : 1184), 2), 256, 0, s>>>(p);
        const int rc = finish_launch();
        if (rc != SPDY_OK) return rc;
    }
    // Widest tile that still gives every multiprocessor one; below that, narrow tiles whose K is shared by a cluster.
    const int64_t tm = (a.M + BM - 1) / BM;
    const int sms = sm_count();
    const int BN = tm * ((a.N + 255) / 256) >= sms ? 256 : tm * ((a.N + 127) / 128) >= sms ? 128 : 64;
    a.tiles_m = static_cast<int>(tm), a.tiles_n = static_cast<int>((a.N + BN - 1) / BN), a.k_blocks = static_cast<int>((a.K + BK - 1) / BK);
    if (tm * a.tiles_n > 0x7fffffff / 8) return SPDY_ERR_UNSUPPORTED;
    int parts = 1;
    while (BN == 64 && parts < 8 && a.tiles_m * a.tiles_n * parts * 2 <= sms && a.k_blocks >= parts * 4) parts *= 2;
    CUtensorMap mx, mw;
    int rc = make_map(&mx, a.x, a.ldx, a.M, a.K, a.dtype, BM);
    if (rc == SPDY_OK) rc = make_map(&mw, a.w, a.ldw, a.N, a.K, a.dtype, BN);
    if (rc != SPDY_OK) return rc;
    if (BN == 256) return launch_tiles<T, 256, ACT>(mx, mw, a, parts, s);
    if (BN == 128) return launch_tiles<T, 128, ACT>(mx, mw, a, parts, s);
    return launch_tiles<T, 64, ACT>(mx, mw, a, parts, s);
}

template <class T, int ROWS, int ACT> int launch_rows_of(const LinearArgs &a, cudaStream_t s)
{
    constexpr int COLS = ROWS == 1 ? 2 : 4;
    const dim3 grid(static_cast<unsigned>((a.N + 4 * COLS - 1) / (4 * COLS)), static_cast<unsigned>((a.M + ROWS - 1) / ROWS));
    if (tma_ok(a.x, a.ldx) && tma_ok(a.w, a.ldw) && a.K % 8 == 0) linear_rows_kernel<T, ROWS, COLS, ACT, true><<<grid, 128, 0, s>>>(a);
    else linear_rows_kernel<T, ROWS, COLS, ACT, false><<<grid, 128, 0, s>>>(a);
    return finish_launch();
}

template <class T, int ACT> int launch_rows(const LinearArgs &a, cudaStream_t s)
{
    if (a.M > 65535 * kFewRows) return SPDY_ERR_UNSUPPORTED;  // K = 0 only
    if (a.M == 1) return launch_rows_of<T, 1, ACT>(a, s);
    if (a.M <= 4) return launch_rows_of<T, 4, ACT>(a, s);
    return launch_rows_of<T, 8, ACT>(a, s);
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

bool half_type(int t) { return t == SPDY_BF16 || t == SPDY_F16; }

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
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return dtype == SPDY_BF16 ? launch_type<__nv_bfloat16>(a, workspace, s) : launch_type<__half>(a, workspace, s);
}

int spdy_linear_check_status(void *cuda_stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    int count = 0;
    const int zero = 0;
    SPDY_EVAL_TRY(cudaMemcpyFromSymbolAsync(&count, g_timeouts, sizeof count, 0, cudaMemcpyDeviceToHost, s));
    SPDY_EVAL_TRY(cudaStreamSynchronize(s));
    if (count == 0) return SPDY_OK;
    SPDY_EVAL_TRY(cudaMemcpyToSymbolAsync(g_timeouts, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, s));
    SPDY_EVAL_TRY(cudaStreamSynchronize(s));
    return SPDY_ERR_INTERNAL;
}

}  // extern "C"
