// What the operators on the tensor cores share (eval_linear.cu, eval_linear_logprobs.cu): barriers, TMA copies and tensor maps, tcgen05
// products and TMEM, pairs of fp32 operations, and copies of operands that TMA cannot read.  Everything has internal linkage.
#ifndef SPDY_EVAL_TENSOR_CUH
#define SPDY_EVAL_TENSOR_CUH

#include <cuda.h>

#include "eval_common.cuh"

namespace spdy_eval {

constexpr int BM = 128, BK = 64;           // rows of a block's tile; a slice of K: 64 16-bit elements = one 128-byte swizzle row

// Waits of this translation unit's kernels that ran out of time (none in a working run); spdy_linear_check_status adds the units' up.
static __device__ int g_timeouts;

// ---------------------------------------------------------------------------------------------- mbarrier, TMA, tcgen05
__device__ __forceinline__ uint32_t smem_addr(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

__device__ __forceinline__ void barrier_init(uint64_t *b, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(b)), "r"(count) : "memory"); }
__device__ __forceinline__ void barrier_arrive(uint64_t *b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(b)) : "memory"); }
__device__ __forceinline__ void barrier_expect(uint64_t *b, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(b)), "r"(bytes) : "memory");
}
// Waits until the phase of `parity` is over; gives up after about two seconds of polling and counts that.
__device__ __forceinline__ bool barrier_wait(uint64_t *b, uint32_t parity)
{
    const uint32_t addr = smem_addr(b);
    Patience patience;
    for (;;) {
        uint32_t done;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(done)
            : "r"(addr), "r"(parity)
            : "memory");
        if (done) return true;
        if (patience.over(clock64())) {
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

// One thread of a converged warp.  The loops below run on whole warps and elect the issuing thread around each TMA or tcgen05
// instruction: these take their operands from uniform registers, and inside a branch on the lane number each operand cost a
// trip there (a pair's 64-wide slice of K: 731 cycles with the branch, 521 this way).
__device__ __forceinline__ bool elect()
{
    uint32_t chosen;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(chosen));
    return chosen != 0;
}
// The address of a shared variable in the first block of the cluster.
__device__ __forceinline__ uint32_t first_blocks(uint32_t addr)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
// Says that what the thread (with tcgen05.fence::before_thread_sync) has read of or written to TMEM is done.  It orders no other memory: with
// release semantics at the cluster's scope the arrival took 1500 to 2200 cycles where stores to global memory were under way.
__device__ __forceinline__ void barrier_arrive_at(uint32_t addr) { asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory"); }
// A copy to this block's shared memory that counts on a barrier of either block of the pair.
__device__ __forceinline__ void tma_load_pair(void *to, const CUtensorMap *map, int x, int y, uint32_t barrier)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_addr(to)),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(barrier)
                 : "memory");
}

template <bool PAIR> __device__ __forceinline__ void tmem_alloc(uint32_t *to, int columns)
{
    if (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(to)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
}
template <bool PAIR> __device__ __forceinline__ void tmem_free(uint32_t tmem, int columns)
{
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
template <bool PAIR> __device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    if (PAIR)
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                     "r"(static_cast<uint32_t>(add))
                     : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc),
                     "r"(static_cast<uint32_t>(add))
                     : "memory");
}
// Signals the barrier (of both blocks of a pair) when the products issued so far are done.
template <bool PAIR> __device__ __forceinline__ void mma_commit(uint64_t *b)
{
    if (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(b)), "h"(static_cast<uint16_t>(3)) : "memory");
    else asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(b)) : "memory");
}
// 16 columns of a warp's 32 rows, a row to a lane.
__device__ __forceinline__ void tmem_load16(uint32_t addr, float *v)
{
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// 32 of them.
__device__ __forceinline__ void tmem_load32(uint32_t addr, float *v)
{
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
        "%28, %29, %30, %31}, [%32];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// 8 of them, added to v.
__device__ __forceinline__ void tmem_add8(uint32_t addr, float *v)
{
    uint32_t r[8];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += __uint_as_float(r[i]);
}

// And back; the warp reads them again only after tmem_stores_wait().
__device__ __forceinline__ void tmem_store32(uint32_t addr, const float *v)
{
    uint32_t r[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(v[i]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, "
        "%28, %29, %30, %31, %32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
        "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_stores_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---------------------------------------------------------------------------------------------- values
// Two fp32 operations per instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<unsigned long long &>(r))
        : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)), "l"(reinterpret_cast<unsigned long long &>(c)));
    return r;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long &>(r)) : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long &>(r)) : "l"(reinterpret_cast<unsigned long long &>(a)), "l"(reinterpret_cast<unsigned long long &>(b)));
    return r;
}
__device__ __forceinline__ void load32(const void *p, uint4 &lo, uint4 &hi)
{
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(lo.x), "=r"(lo.y), "=r"(lo.z), "=r"(lo.w), "=r"(hi.x), "=r"(hi.y), "=r"(hi.z), "=r"(hi.w)
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store32(void *p, uint4 lo, uint4 hi)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(lo.x), "r"(lo.y), "r"(lo.z), "r"(lo.w), "r"(hi.x), "r"(hi.y), "r"(hi.z), "r"(hi.w)
                 : "memory");
}


// ---------------------------------------------------------------------------------------------- operands
// Copies of operands whose rows TMA cannot read (a row has to start on 16 bytes), with rows of ldto elements.  They cost one more
// read and write of such an operand and a launch (both unaligned, in a graph: 333 x 1001 x 517 10.9 us, 2048 x 4096 x 1001 24.9).
struct Repack {
    const uint16_t *from[2];
    uint16_t *to[2];
    int64_t ld[2], rows[2], K, ldto;
};
// A thread copies eight elements of a row at a time, from the two aligned blocks of 16 bytes around them where these lie inside the matrix,
// and two such copies together, which keeps more loads under way.  What lies behind K is whatever (TMA never reads it).  50001 rows of
// 1000 elements, an odd stride: 31 us, 6.4 TB/s (53 us with words of 4 bytes; 43 with the parameters not in constant memory, which
// `which` indexes, but copied by each thread; one copy at a time cost 6 us more than two, four as much as two).
constexpr int kRepackBlock = 512;  // copies
// I: a division by a 64-bit number costs more than the copy, so it is done where the copies pass 32 bits only.
template <class I> __global__ void __launch_bounds__(256) repack_kernel(const __grid_constant__ Repack p)
{
    constexpr int kAtOnce = kRepackBlock / 256;
    const int which = blockIdx.y;
    if (!p.to[which]) return;
    const I per_row = static_cast<I>(p.ldto / 8), total = static_cast<I>(p.rows[which]) * per_row;
    const int64_t ld = p.ld[which];
    const uint16_t *const matrix = p.from[which];
    const uintptr_t first = reinterpret_cast<uintptr_t>(matrix), end = first + static_cast<uint64_t>((p.rows[which] - 1) * ld + p.K) * 2;
    for (I i0 = static_cast<I>(blockIdx.x) * kRepackBlock + threadIdx.x; i0 < total; i0 += static_cast<I>(gridDim.x) * kRepackBlock) {
        uint4 a[kAtOnce], b[kAtOnce];
        const uint16_t *from[kAtOnce];
        int64_t place[kAtOnce];
        int left[kAtOnce];
        bool inside[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const I i = i0 + u * 256;
            const int64_t r = i / per_row, k = static_cast<int64_t>(i - static_cast<I>(r) * per_row) * 8;
            from[u] = matrix + r * ld + k, place[u] = r * p.ldto + k;
            left[u] = i < total ? static_cast<int>(min(p.K - k, static_cast<int64_t>(8))) : 0;
            const uintptr_t at = reinterpret_cast<uintptr_t>(from[u]) & ~static_cast<uintptr_t>(15);
            inside[u] = at >= first && at + 32 <= end;
            a[u] = b[u] = make_uint4(0, 0, 0, 0);
            if (left[u] > 0 && inside[u]) a[u] = *reinterpret_cast<const uint4 *>(at), b[u] = *reinterpret_cast<const uint4 *>(at + 16);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (left[u] <= 0) continue;
            const uintptr_t at = reinterpret_cast<uintptr_t>(from[u]);
            uint32_t v[8] = {a[u].x, a[u].y, a[u].z, a[u].w, b[u].x, b[u].y, b[u].z, b[u].w}, w[4];
#pragma unroll
            for (int j = 0; j < 6; ++j) v[j] = at & 8 ? v[j + 2] : v[j];
#pragma unroll
            for (int j = 0; j < 5; ++j) v[j] = at & 4 ? v[j + 1] : v[j];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = __funnelshift_r(v[j], v[j + 1], at & 2 ? 16 : 0);
            if (!inside[u])
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t lo = 2 * j < left[u] ? from[u][2 * j] : 0, hi = 2 * j + 1 < left[u] ? from[u][2 * j + 1] : 0;
                    w[j] = lo | hi << 16;
                }
            *reinterpret_cast<uint4 *>(p.to[which] + place[u]) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

// Both copies, where there are any.
static inline int repack(const Repack &p, cudaStream_t s)
{
    if (!p.to[0] && !p.to[1]) return SPDY_OK;
    constexpr int64_t most = 148 * 16;
    const int64_t rows = p.rows[0] > p.rows[1] ? p.rows[0] : p.rows[1], copies = rows * (p.ldto / 8), want = (copies + kRepackBlock - 1) / kRepackBlock;
    const dim3 grid(static_cast<unsigned>(want < most ? want : most), 2);
    if (copies + (most + 1) * kRepackBlock < (1ll << 32)) repack_kernel<uint32_t><<<grid, 256, 0, s>>>(p);
    else repack_kernel<uint64_t><<<grid, 256, 0, s>>>(p);
    return finish_launch();
}

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static inline EncodeTiled encode_tiled()
{
    static EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

static inline int make_map(CUtensorMap *map, const void *p, int64_t ld, int64_t rows, int64_t K, int dtype, int box_rows)
{
    EncodeTiled encode = encode_tiled();
    if (!encode) return SPDY_ERR_UNSUPPORTED;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(K), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(ld) * 2};
    const cuuint32_t box[2] = {BK, static_cast<cuuint32_t>(box_rows)}, steps[2] = {1, 1};
    const CUresult rc = encode(map, dtype == SPDY_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void *>(p), dims, strides, box,
                               steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return rc == CUDA_SUCCESS ? SPDY_OK : SPDY_ERR_UNSUPPORTED;
}

static inline bool tma_ok(const void *p, int64_t ld) { return aligned(p, 16) && ld % 8 == 0 && ld * 2 < (1ll << 40); }
static inline int64_t packed_ld(int64_t K) { return (K + 7) / 8 * 8; }
static inline size_t packed_bytes(int64_t rows, int64_t K) { return (static_cast<size_t>(rows) * static_cast<size_t>(packed_ld(K)) * 2 + 255) / 256 * 256; }

static inline bool half_type(int t) { return t == SPDY_BF16 || t == SPDY_F16; }


// Reads and clears this translation unit's count of waits that ran out, waiting for the stream.
static inline int take_timeouts(cudaStream_t s, int *count)
{
    const int zero = 0;
    *count = 0;
    SPDY_EVAL_TRY(cudaMemcpyFromSymbolAsync(count, g_timeouts, sizeof *count, 0, cudaMemcpyDeviceToHost, s));
    SPDY_EVAL_TRY(cudaStreamSynchronize(s));
    if (*count == 0) return SPDY_OK;
    SPDY_EVAL_TRY(cudaMemcpyToSymbolAsync(g_timeouts, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, s));
    SPDY_EVAL_TRY(cudaStreamSynchronize(s));
    return SPDY_OK;
}

}  // namespace spdy_eval
#endif
