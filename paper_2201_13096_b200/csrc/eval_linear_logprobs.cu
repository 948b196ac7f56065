// Log probabilities of given tokens under softmax((hidden weight^T + bias) / T), entropy and gradients, without a table of logits:
// kernels and C entries (spdy_eval.h).
//
// Everything large is a product on the tensor cores, carried by one kernel: pairs of multiprocessors (cta_group::2) on tiles of
// 256 x 256, operands brought by TMA, two fp32 accumulators in TMEM, sixteen warps that carry a finished tile on while the next
// is multiplied.  What is done with a tile differs:
//   kStats   logits of 256 rows and ids -> per row the largest, the sum of exponentials relative to it, and the sum that the
//            entropy needs; the given token's logit.  A second kernel joins a row's tiles in their order.
//   kLogits  the same, and the logits are kept, in 16 bits as logarithms relative to the largest of 32, for a kernel that turns them into the
//            gradient by them in place
//   kGrad    the logits once more -> the gradient by them, rounded to 16 bits
//   kHidden  gradient x weight: fp32 sums of dhidden
//   kWeight  gradient^T x hidden: dweight (kWeightParts: as fp32 sums)
// Two plans keep what is of size rows x ids within a budget.  By ids (a backward call, whose sums are known, and narrow heads): the
// gradient of all rows for a piece of the vocabulary at a time, dhidden added up over the pieces; the logits are multiplied again.
// By rows (the rest of the calls that give values and gradients at once): the logits of some rows and all ids at a time, dweight added up over them; each
// product is done once.  In the last two products one or both operands have the summed index as their rows ("MN-major"); TMA brings
// them as boxes of 64 columns, and the matrix descriptors name that order, so nothing is transposed.
#include <limits.h>

#include "eval_tensor.cuh"

using namespace spdy_eval;

namespace spdy_eval {
int linear_logprobs_timeouts(cudaStream_t s, int *count) { return take_timeouts(s, count); }
}

namespace {

namespace cg = cooperative_groups;

constexpr int kSlices = 2;                               // 64-wide slices of the summed index to a stage
constexpr int kTile = 256, kWarpColumns = 64;            // of a pair's tile; columns that an epilogue warp carries
constexpr int kEpilogueWarps = 16, kThreads = 32 * (2 + kEpilogueWarps);
constexpr int kSliceBytes = 2 * BM * BK * 2;             // 128 rows or columns of each operand
constexpr int kStageBytes = kSlices * kSliceBytes, kStages = 196608 / kStageBytes;
constexpr int kStageK = kSlices * BK;
constexpr int kConsts = 8;                               // floats per row that the gradient needs

// A call's kernels follow one another by programmatic launches: each is set up while the one before still runs, waits for its end here
// before it touches memory, and lets the next one in.
__device__ __forceinline__ void wait_for_previous()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// The tensor core cuts its partial sums towards 0 where fp32 additions would round: a sum of many products ends short of itself, by how much
// depends on the data.  The sums that logits are go into several accumulators therefore, a few stages to each, which the epilogue adds up in fp32.
// How far lse is off, relative, at widths 256 to 16384 (positive products in half precision): 2 stages each 1.7e-7 to 2.8e-7 (7e-7), first 3, 3, then 2
// 1.8e-7 to 4.1e-7 (7e-7 to 1.2e-6), 4 each 2.0e-7 to 4.8e-7 (1.6e-6), all in one 2.2e-6 at 2624 already (the plain fp32 form 0.8e-7 to 1.2e-6).
// Values of 4096 x 16384 x 1024: 107, 97, 90 and 89 us.  The first two are longer because the next tile's have to keep the tensor cores busy while the
// epilogue is still at work on this one.
struct Pieces {
    int first, rest;  // stages of the first two pieces, and of each that follows
};
constexpr Pieces kLogitPieces = {3, 2}, kGradPieces = {4, 4};

enum Kind { kStats, kLogits, kGrad, kHidden, kWeight, kWeightParts };

// Which operands have the summed index as their rows.
template <int KIND> struct Order {
    static constexpr bool kA = KIND == kWeight || KIND == kWeightParts, kB = kA || KIND == kHidden;
};
template <int KIND> constexpr bool kInPieces = KIND == kStats || KIND == kLogits || KIND == kGrad;

struct ProductArgs {
    int64_t M, N;                  // rows and columns of the result that exist
    Tiles tiles;                   // of the result
    int splits, k_blocks;          // shares of the summed index, its stages
    Divisor per_split;
    int a_row0, b_row0;            // first rows of the operands
    // kStats, kGrad
    const void *bias, *tokens;
    int bias_type, index_bits;
    int64_t v0;                    // the first column's id
    float c;                       // log2(e) / T
    Pieces pieces;
    float *partial, *token_logit;  // [tiles_n][3][padded_rows], [M]
    int64_t padded_rows;
    const float *consts;           // [M][kConsts]
    const uint32_t *scale_bits;    // NULL, or the largest gradient's bits (half precision)
    float *column_sums;            // NULL, or [row groups of 32][N]
    int64_t ld_sums;
    uint8_t *fine;                 // kLogits: NULL, or the codes' lower bits, [M][ldo]
    float *tops;                   // kLogits: [ids / 32][padded_rows], what a row's 32 codes are relative to
    int low;                       // kGrad: 0, or the row of the piece from which the lower halves lie,
    int64_t below;                 // that many bytes behind the upper ones (as a product of the two in the kernel it was kept in registers throughout)
    int wrap;                      // products over rows: from this one on the second operand's begin again
    void *out;                     // kLogits: codes; kGrad: the piece; kWeight: 16 bits; parts: fp32 [splits][M][ldo]
    int64_t ldo;
    const float *sums;             // kWeight: NULL, or fp32 [M][ld_old] to add
    int64_t ld_old;
    int add, width;                // parts: to what is there already; kWeight: 32 or 16 if every row of out starts on as many bytes, else 0
};

// Half precision keeps the gradient by the logits times a power of two that brings the largest row's to 2^13 .. 2^14: the least normal number is then
// 2^-28 of it.
__device__ __forceinline__ int scale_power(const uint32_t *bits)
{
    if (!bits) return 0;
    const int e = static_cast<int>(*bits >> 23);
    return e == 0 || e >= 255 ? 0 : min(13 - (e - 127), 100);
}
__device__ __forceinline__ float power_of_two(int k) { return __int_as_float((k + 127) << 23); }

__device__ __forceinline__ int64_t token_at(const void *tokens, int bits, int64_t r)
{
    return bits == 64 ? static_cast<const int64_t *>(tokens)[r] : static_cast<const int32_t *>(tokens)[r];
}
__device__ __forceinline__ float value_at(const void *p, int type, int64_t n)
{
    if (type == SPDY_F32) return static_cast<const float *>(p)[n];
    if (type == SPDY_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[n]);
    return __half2float(static_cast<const __half *>(p)[n]);
}

// Running sums of a row relative to its largest logit m: s = sum 2^((x - m) c), t = sum 2^((x - m) c) (x - m) c.
struct Sums {
    float m, s, t;
};
// Relative to `top` >= m instead.  A shift beyond -1e30 leaves nothing, and is cut there so that 0 times it stays 0.
__device__ __forceinline__ void raise(Sums &a, float top, float c)
{
    if (a.s != 0.f) {
        const float shift = max_nan((a.m - top) * c, -1e30f), f = ex2(shift);
        a.t = f * fmaf(a.s, shift, a.t);
        a.s *= f;
    }
    a.m = top;
}
__device__ __forceinline__ void join(Sums &a, Sums b, float c)
{
    const float top = fmaxf(a.m, b.m);
    raise(a, top, c), raise(b, top, c);
    a.s += b.s, a.t += b.t;
}

// Descriptor of an operand whose rows are the summed index: boxes of 64 columns (128 bytes, swizzled) and 64 rows, 8 KB apart;
// groups of 8 rows lie 1024 bytes apart.
__device__ __forceinline__ uint64_t operand_by_columns(uint32_t addr)
{
    return static_cast<uint64_t>((addr & 0x3ffffu) >> 4) | 512ull << 16 | 64ull << 32 | 1ull << 46 | 2ull << 61;
}

struct Control {
    uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
};

// Adds 32 logits, of which `top` is at least the largest, to the sums, which become relative to it.  `each` gets (x - top) c by pairs.
template <class Each> __device__ __forceinline__ void add_exponentials(const float *f, float top, float c, Sums &sums, Each each)
{
    raise(sums, top, c);
    const float2 from = both(top == neg_inf() ? 0.f : -top), cc = both(c);  // first the difference, so that logits of any size keep their digits
    float2 s = both(0.f), t = both(0.f);
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float2 d = mul2(add2(make_float2(f[i], f[i + 1]), from), cc);
        d = make_float2(max_nan(d.x, -200.f), max_nan(d.y, -200.f));  // below, the exponential is 0
        const float2 e = make_float2(ex2(d.x), ex2(d.y));
        s = add2(s, e);
        t = fma2(e, d, t);
        each(i, d);
    }
    sums.s += s.x + s.y, sums.t += t.x + t.y;
}

// ---------------------------------------------------------------------------------------------- what is done with a tile
// Each function carries 64 columns of a warp's 32 rows, a row to a lane.  `ready` waits for the accumulator and says whether it came
// (if not, what is written is NaN), and only then is `tmem` where it lies; `release` is called once the last columns have left TMEM.

// The ids' bias in the warp's shared memory.
__device__ __forceinline__ void stage_bias(const ProductArgs &a, int64_t n0, float *bias)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
    for (int i = lane; i < kWarpColumns; i += 32) bias[i] = a.bias && n0 + i < a.N ? value_at(a.bias, a.bias_type, a.v0 + n0 + i) : 0.f;
    __syncwarp();
}
// 32 logits of a row; ids beyond the vocabulary are -inf.
__device__ __forceinline__ void load_logits(const ProductArgs &a, uint32_t tmem, int64_t n, const float *bias, float *f)
{
    tmem_load32(tmem, f);
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float4 b = reinterpret_cast<const float4 *>(bias)[i];
            const float2 lo = add2(make_float2(f[4 * i], f[4 * i + 1]), make_float2(b.x, b.y)), hi = add2(make_float2(f[4 * i + 2], f[4 * i + 3]), make_float2(b.z, b.w));
            f[4 * i] = lo.x, f[4 * i + 1] = lo.y, f[4 * i + 2] = hi.x, f[4 * i + 3] = hi.y;
        }
    }
    if (n + 32 > a.N)
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (n + i >= a.N) f[i] = neg_inf();
}
// f[at], for a row in which it is one of the 32.
__device__ __forceinline__ float pick(const float *f, int64_t at)
{
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) x = at == i ? f[i] : x;
    return x;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ float largest(const float *f, float top)
{
    float other = f[0];
#pragma unroll
    for (int i = 1; i + 4 <= 32; i += 4) top = max3(top, f[i], f[i + 1]), other = max3(other, f[i + 2], f[i + 3]);
    return fmaxf(max3(top, f[29], f[30]), fmaxf(other, f[31]));
}

template <class Ready, class Release>
__device__ __forceinline__ Sums carry_stats(const ProductArgs &a, const uint32_t &tmem, int64_t m, int64_t n0, float *bias, Ready ready, Release release)
{
    int64_t token = -1;
    if (m < a.M && a.token_logit) token = token_at(a.tokens, a.index_bits, m);
    stage_bias(a, n0, bias);
    if (!ready()) {
        if (token >= n0 && token < n0 + kWarpColumns && token < a.N) a.token_logit[m] = quiet_nan();
        return {0.f, quiet_nan(), quiet_nan()};
    }
    Sums sums = {neg_inf(), 0.f, 0.f};
#pragma unroll 1
    for (int c = 0; c < kWarpColumns; c += 32) {
        float f[32];
        load_logits(a, tmem + c, n0 + c, bias + c, f);
        if (c + 32 == kWarpColumns) release();
        const int64_t at = token - (n0 + c);
        if (at >= 0 && at < 32 && token < a.N) a.token_logit[m] = pick(f, at);
        add_exponentials(f, largest(f, sums.m), a.c, sums, [](int, float2) {});
    }
    return sums;
}

// A kept logit: how far log2 of its exponential lies below that of the largest among 32 ids, in steps of 2^-10
// octaves over 64 octaves for bf16, 2^-11 over 32 for half precision, whose own numbers end sooner.  p comes out within 2^-11 ln 2 =
// 3.4e-4 of itself (1.7e-4), beside the 16-bit rounding that follows of 3.9e-3 (4.9e-4).  The last code is "nothing".
// FINE, where dbias wants p to fp32's digits: another 7 bits, in bytes of their own.
template <class T> constexpr float kSteps = std::is_same<T, __nv_bfloat16>::value ? 1024.f : 2048.f;
constexpr uint32_t kNothing = 65535;
template <class T, bool FINE> constexpr float kCodeSteps = kSteps<T> * (FINE ? 128.f : 1.f);
template <bool FINE> constexpr float kLastCode = FINE ? 8388607.f : 65535.f;

// As carry_stats, with the codes, and per 32 of them the largest, which they are relative to.
constexpr int kCodes = 32;
template <class T, bool FINE, class Ready, class Release>
__device__ __forceinline__ Sums carry_logits(const ProductArgs &a, const uint32_t &tmem, int64_t m, int64_t n0, float *bias, Ready ready, Release release)
{
    int64_t token = -1;
    if (m < a.M && a.token_logit) token = token_at(a.tokens, a.index_bits, m);
    stage_bias(a, n0, bias);
    if (!ready()) {
        if (token >= n0 && token < n0 + kWarpColumns && token < a.N) a.token_logit[m] = quiet_nan();
        return {0.f, quiet_nan(), quiet_nan()};  // the row's sum is NaN, and with it all that comes of its codes
    }
    Sums sums = {neg_inf(), 0.f, 0.f};
    uint16_t *to = static_cast<uint16_t *>(a.out) + m * a.ldo + n0;
#pragma unroll 1
    for (int c = 0; c < kWarpColumns; c += kCodes) {
        float f[kCodes];
        load_logits(a, tmem + c, n0 + c, bias + c, f);
        if (c + kCodes == kWarpColumns) release();
        const int64_t at = token - (n0 + c);
        if (at >= 0 && at < kCodes && token < a.N) a.token_logit[m] = pick(f, at);
        const float top = largest(f, neg_inf());
        Sums here = {neg_inf(), 0.f, 0.f};
        uint32_t w[kCodes / 2], low[FINE ? kCodes / 4 : 1];
        add_exponentials(f, top, a.c, here, [&](int i, float2 d) {
            // 2^23 and a number below it: rounded to a whole number, in the lower part of the pattern
            constexpr float lowest = -kLastCode<FINE> / kCodeSteps<T, FINE>;
            const float2 code = fma2(make_float2(fmaxf(d.x, lowest), fmaxf(d.y, lowest)), both(-kCodeSteps<T, FINE>), both(8388608.f));
            const uint32_t x = __float_as_uint(code.x), y = __float_as_uint(code.y);
            w[i / 2] = FINE ? __byte_perm(x >> 7, y >> 7, 0x5410) : __byte_perm(x, y, 0x5410);
            if (FINE) {
                const uint32_t two = __byte_perm(x, y, 0x0040) & 0x7f7fu;
                if (i % 4 == 0) low[i / 4] = two;
                else low[i / 4] |= two << 16;
            }
        });
        if (m < a.M && n0 + c < a.N) {  // ldo is a multiple of 64
            a.tops[(n0 + c) / kCodes * a.padded_rows + m] = top;
            store32(to + c, make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7]));
            store32(to + c + 16, make_uint4(w[8], w[9], w[10], w[11]), make_uint4(w[12], w[13], w[14], w[15]));
            if constexpr (FINE) store32(a.fine + m * a.ldo + n0 + c, make_uint4(low[0], low[1], low[2], low[3]), make_uint4(low[4], low[5], low[6], low[7]));
        }
        join(sums, here, a.c);
    }
    return sums;
}

// Sums over the 32 rows of 16 columns, each lane's `f`: of column `lane / 2` in the lane, by halves of the columns that partners exchange.
__device__ __forceinline__ float sum_columns(const float *f)
{
    const int lane = threadIdx.x & 31;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool up = lane & 16;
        v[i] = (up ? f[i + 8] : f[i]) + __shfl_xor_sync(0xffffffffu, up ? f[i] : f[i + 8], 16);
    }
#pragma unroll
    for (int half = 4, bit = 8; half; half >>= 1, bit >>= 1) {
        const bool up = lane & bit;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < half) v[i] = (up ? v[i + half] : v[i]) + __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + half], bit);
    }
    return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}

// What the gradient by a row's logits needs: d = [v = token] hit - p (all + slope y), y = log2 p = (x - ref) c - ls; `known` is d at the
// token, from its logit in fp32: where the logits are kept in fewer bits, 1 - p of a token that is all but certain would be lost.
struct RowConsts {
    float ref, ls, hit, all, slope;
    int token;
    float known;
};
__device__ __forceinline__ RowConsts row_consts(const float *consts, int64_t m, float scale)
{
    const float4 k = reinterpret_cast<const float4 *>(consts)[2 * m], more = reinterpret_cast<const float4 *>(consts)[2 * m + 1];
    return {k.x, k.y, k.z * scale, k.w * scale, more.x * scale, __float_as_int(more.y), more.z * scale};
}
// -p (all + slope y).  ENT: with the entropy's gradient (slope is not 0); below -200 p is 0.
template <bool ENT> __device__ __forceinline__ float grad_at(float y, const RowConsts &k)
{
    y = min_nan(y, 0.f);
    return ENT ? -ex2(y) * fmaf(k.slope, max_nan(y, -200.f), k.all) : -ex2(y) * k.all;
}

// What rounding to 16 bits takes from numbers, in 16 bits; nothing of ones that are not finite in them.
template <class T> __device__ __forceinline__ uint4 lower_halves(const float *f, uint4 rounded)
{
    float r[8];
    Elem<T>::unpack(rounded, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = fabsf(r[i]) <= 3.39e38f ? f[i] - r[i] : 0.f;
    return Elem<T>::pack(r);
}

// Gradient by 64 logits of a row, rounded to 16 bits once (or in two halves).
template <class T, bool ENT, class Ready, class Release>
__device__ __forceinline__ void carry_grad(const ProductArgs &a, const uint32_t &tmem, int64_t m0, int64_t n0, float *bias, Ready ready, Release release)
{
    const int lane = threadIdx.x & 31;
    const int64_t m = m0 + lane;
    const bool inside = m < a.M;
    if (inside) asm volatile("prefetch.global.L1 [%0];" ::"l"(a.consts + static_cast<int64_t>(m) * kConsts));  // no registers for them while sums are added up
    stage_bias(a, n0, bias);
    const bool ok = ready();
    RowConsts k = {0.f, 0.f, 0.f, 0.f, 0.f, -1, 0.f};
    if (inside) k = row_consts(a.consts, m, power_of_two(scale_power(a.scale_bits)));
    char *to = static_cast<char *>(a.out) + (m * a.ldo + n0) * 2;
#pragma unroll 1
    for (int c = 0; c < kWarpColumns; c += 32) {
        float f[32];
        load_logits(a, tmem + c, n0 + c, bias + c, f);
        if (c + 32 == kWarpColumns) release();
        if (n0 + c >= a.N) continue;
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
            const float2 y = fma2(add2(make_float2(f[i], f[i + 1]), both(-k.ref)), both(a.c), both(-k.ls));
            f[i] = grad_at<ENT>(y.x, k), f[i + 1] = grad_at<ENT>(y.y, k);
        }
        const int64_t at = k.token - (a.v0 + n0 + c);
        if (at >= 0 && at < 32)
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (at == i) f[i] += k.hit;
        if (!ok)
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = quiet_nan();
        if (inside) {  // ldo is a multiple of 64
#pragma unroll
            for (int i = 0; i < 32; i += 16) {
                const uint4 x = Elem<T>::pack(f + i), y = Elem<T>::pack(f + i + 8);
                store32(to + 2 * (c + i), x, y);
                if (a.low) store32(to + a.below + 2 * (c + i), lower_halves<T>(f + i, x), lower_halves<T>(f + i + 8, y));
            }
        } else if (m < a.low) {
#pragma unroll
            for (int i = 0; i < 32; i += 16) store32(to + 2 * (c + i), make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0));
        }
        if (a.column_sums) {
            if (!inside)
#pragma unroll
                for (int i = 0; i < 32; ++i) f[i] = 0.f;
#pragma unroll
            for (int i = 0; i < 32; i += 16) {
                const float sum = sum_columns(f + i);
                const int64_t n = n0 + c + i + (lane >> 1);
                if (!(lane & 1) && n < a.N && m0 < a.M) a.column_sums[m0 / 32 * a.ld_sums + n] = sum;
            }
        }
    }
}

template <class Ready, class Release>
__device__ __forceinline__ void carry_parts(const ProductArgs &a, uint32_t tmem, int split, int64_t m0, int64_t n0, Ready ready, Release release)
{
    const int64_t m = m0 + (threadIdx.x & 31);
    float *to = static_cast<float *>(a.out) + (split * a.M + m) * a.ldo + n0;
    const bool ok = ready();
#pragma unroll 1
    for (int c = 0; c < kWarpColumns; c += 16) {
        float f[16];
        tmem_load16(tmem + c, f);
        if (c + 16 == kWarpColumns) release();
        if (m >= a.M) continue;
#pragma unroll
        for (int h = 0; h < 16; h += 8) {
            if (n0 + c + h >= a.N) break;  // ldo is a multiple of 8
            uint4 lo, hi;
            float old[8] = {};
            if (a.add) load32(to + c + h, lo, hi), Elem<float>::unpack(lo, old), Elem<float>::unpack(hi, old + 4);
#pragma unroll
            for (int i = 0; i < 8; ++i) old[i] = ok ? old[i] + f[h + i] : quiet_nan();
            store32(to + c + h, Elem<float>::pack(old), Elem<float>::pack(old + 4));
        }
    }
}

// 16 columns (from n) of 32 rows (from m), a row to a lane, stored by runs of columns; 1 KB of shared memory of the warp's own.
__device__ __noinline__ void store_turned(const ProductArgs &a, int64_t m, int64_t n, uint4 v0, uint4 v1, unsigned char *turn)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
    reinterpret_cast<uint4 *>(turn)[2 * lane] = v0;
    reinterpret_cast<uint4 *>(turn)[2 * lane + 1] = v1;
    __syncwarp();
    uint16_t *y = static_cast<uint16_t *>(a.out);
#pragma unroll
    for (int it = 0; it < 16; ++it) {
        const int64_t row = m + it * 2 + lane / 16, col = n + lane % 16;
        if (row < a.M && col < a.N) y[row * a.ldo + col] = reinterpret_cast<const uint16_t *>(turn)[it * 32 + lane];
    }
}

template <class T, class Ready, class Release>
__device__ __forceinline__ void carry_store(const ProductArgs &a, uint32_t tmem, int64_t m0, int64_t n0, unsigned char *turn, Ready ready, Release release)
{
    const int64_t m = m0 + (threadIdx.x & 31);
    char *to = static_cast<char *>(a.out) + (m * a.ldo + n0) * 2;
    const float scale = power_of_two(-scale_power(a.scale_bits));
    const bool ok = ready();
#pragma unroll 1
    for (int c = 0; c < kWarpColumns; c += 16) {
        float f[16];
        tmem_load16(tmem + c, f);
        if (c + 16 == kWarpColumns) release();
        if (n0 + c >= a.N) continue;
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] = ok ? f[i] : quiet_nan();
        if (a.sums && m < a.M) {
            const float *from = a.sums + m * a.ld_old + n0 + c;
#pragma unroll
            for (int h = 0; h < 16; h += 8) {
                if (n0 + c + h >= a.N) break;  // ld_old is a multiple of 8
                uint4 x, y;
                float old[8];
                load32(from + h, x, y);
                Elem<float>::unpack(x, old), Elem<float>::unpack(y, old + 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[h + i] += old[i];
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) f[i] *= scale;
        const uint4 lo = Elem<T>::pack(f), hi = Elem<T>::pack(f + 8);
        if (!a.width || n0 + c + 16 > a.N) {
            store_turned(a, m0, n0 + c, lo, hi, turn);
        } else if (m < a.M) {
            if (a.width == 32) store32(to + 2 * c, lo, hi);
            else reinterpret_cast<uint4 *>(to + 2 * c)[0] = lo, reinterpret_cast<uint4 *>(to + 2 * c)[1] = hi;
        }
    }
}

// ---------------------------------------------------------------------------------------------- the product
constexpr int kBiasBytes = kEpilogueWarps * kWarpColumns * 4, kTurnBytes = kEpilogueWarps * 1024, kJoinBytes = 2 * 16 * 32 * 12;
template <int KIND> constexpr int extra_bytes() { return KIND == kStats || KIND == kLogits ? kBiasBytes + kJoinBytes : KIND == kGrad ? kBiasBytes : KIND == kWeight ? kTurnBytes : 0; }
template <int KIND> constexpr int smem_bytes() { return 1024 + kStages * kStageBytes + extra_bytes<KIND>(); }

// ENT: kGrad with the entropy's gradient; kLogits with the codes' lower bits.
template <class T, int KIND, bool ENT>
__global__ void __launch_bounds__(kThreads, 1) product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ ProductArgs a)
{
    extern __shared__ unsigned char raw_smem[];
    unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~static_cast<uintptr_t>(1023));
    unsigned char *extra = stages + kStages * kStageBytes;
    __shared__ Control ctl;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    cg::cluster_group cluster = cg::this_cluster();
    const int part = static_cast<int>(cluster.block_rank());
    const int items = static_cast<int>(a.tiles.count()) * a.splits, first = static_cast<int>(blockIdx.x) / 2, step = static_cast<int>(gridDim.x) / 2;
    constexpr bool kColumnsA = Order<KIND>::kA, kColumnsB = Order<KIND>::kB;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) barrier_init(&ctl.full[i], 1), barrier_init(&ctl.empty[i], 1);
        for (int i = 0; i < 2; ++i) barrier_init(&ctl.acc_full[i], 1), barrier_init(&ctl.acc_empty[i], 2 * kEpilogueWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_a)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_b)) : "memory");
    }
    __syncwarp();
    if (warp == 1) tmem_alloc<true>(&ctl.tmem, 512);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster.sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = ctl.tmem;
    wait_for_previous();
    const auto range = [&](int split, int &kb0, int &kb1) {
        kb0 = 0, kb1 = a.k_blocks;
        if (KIND == kHidden || KIND == kWeightParts)  // below 2^24 stages, up to 64 shares
            kb0 = static_cast<int>(a.per_split.of(static_cast<uint32_t>(a.k_blocks) * split)), kb1 = static_cast<int>(a.per_split.of(static_cast<uint32_t>(a.k_blocks) * (split + 1)));
    };

    if (warp == 0) {
        int stage = 0, issued = 0;
        uint32_t parity = 0;
        bool ok = true;
        for (int item = first; item < items && ok; item += step) {
            int split, tm, tn, kb0, kb1;
            a.tiles.at(static_cast<uint32_t>(item), split, tm, tn);
            range(split, kb0, kb1);
            const int m0 = tm * kTile + part * BM, n0 = tn * kTile + part * BM;
            if (kb0 == kb1) continue;  // a share of the last, shorter piece may be empty: nothing to add
            for (int kb = kb0; kb < kb1; ++kb) {
                ok = __all_sync(0xffffffffu, barrier_wait(&ctl.empty[stage], parity ^ 1));
                if (!ok) break;
                unsigned char *to = stages + stage * kStageBytes;
                if (elect()) {
                    const uint32_t full = first_blocks(smem_addr(&ctl.full[stage]));  // both blocks' copies count on the first block's barrier
                    if (part == 0) barrier_expect(&ctl.full[stage], 2 * kStageBytes);
#pragma unroll
                    for (int q = 0; q < kSlices; ++q) {
                        const int k = (kb * kSlices + q) * BK;
                        unsigned char *ta = to + q * kSliceBytes, *tb = ta + BM * BK * 2;
                        if (kColumnsA) tma_load_pair(ta, &map_a, m0, k, full), tma_load_pair(ta + 8192, &map_a, m0 + 64, k, full);
                        else tma_load_pair(ta, &map_a, k, a.a_row0 + m0, full);
                        const int row = a.b_row0 + (kColumnsA && k >= a.wrap ? k - a.wrap : k);
                        if (kColumnsB) tma_load_pair(tb, &map_b, n0, row, full), tma_load_pair(tb + 8192, &map_b, n0 + 64, row, full);
                        else tma_load_pair(tb, &map_b, k, a.b_row0 + n0, full);
                    }
                }
                __syncwarp();
                ++issued;
                if (++stage == kStages) stage = 0, parity ^= 1;
            }
        }
        // no copy outlives the block, whatever the other warps met (both blocks' are counted on the first one's barriers)
        if (part == 0)
            for (int i = 0; i < kStages && i < issued; ++i) {
                const int n = issued - 1 - i;
                barrier_wait(&ctl.full[n % kStages], n / kStages & 1);
            }
    } else if (warp == 1) {
        if (part == 0) {
            constexpr uint32_t format = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
            constexpr uint32_t idesc = 1u << 4 | format << 7 | format << 10 | static_cast<uint32_t>(kColumnsA) << 15 | static_cast<uint32_t>(kColumnsB) << 16 |
                                       static_cast<uint32_t>(kTile / 8) << 17 | static_cast<uint32_t>(kTile / 16) << 24;
            int stage = 0, acc = 0, issued = 0;
            uint32_t parity = 0, acc_parity = 0;
            bool ok = true;
            for (int item = first; item < items && ok; item += step) {
                int split, tm, tn, kb0, kb1;
                a.tiles.at(static_cast<uint32_t>(item), split, tm, tn);
                range(split, kb0, kb1);
                if (kb0 == kb1) continue;
                uint32_t d = 0;
                for (int kb = kb0, left = 0, piece = 0; kb < kb1; ++kb) {
                    const bool begins = left == 0;
                    if (begins) left = kInPieces<KIND> ? min(kb1 - kb, piece < 2 ? a.pieces.first : a.pieces.rest) : kb1 - kb, ++piece;
                    const bool ends = --left == 0;
                    if (begins) {
                        ok = __all_sync(0xffffffffu, barrier_wait(&ctl.acc_empty[acc], acc_parity ^ 1));
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        d = tmem + acc * kTile;
                    }
                    ok = __all_sync(0xffffffffu, barrier_wait(&ctl.full[stage], parity));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t at = smem_addr(stages + stage * kStageBytes);
                    if (elect()) {
#pragma unroll
                        for (int q = 0; q < kSlices; ++q) {
                            const uint32_t pa = at + q * kSliceBytes, pb = pa + BM * BK * 2;
                            const uint64_t da = kColumnsA ? operand_by_columns(pa) : operand(pa), db = kColumnsB ? operand_by_columns(pb) : operand(pb);
                            // 16 of the summed index further: 32 bytes along a row, or 16 rows of 128 bytes
#pragma unroll
                            for (int k = 0; k < BK / 16; ++k) mma<true>(d, da + (kColumnsA ? 128 : 2) * k, db + (kColumnsB ? 128 : 2) * k, idesc, !begins || q > 0 || k > 0);
                        }
                        mma_commit<true>(&ctl.empty[stage]);
                        if (ends) mma_commit<true>(&ctl.acc_full[acc]);
                    }
                    __syncwarp();
                    ++issued;
                    if (++stage == kStages) stage = 0, parity ^= 1;
                    if (ends && ++acc == 2) acc = 0, acc_parity ^= 1;
                }
            }
            // nor does a product: TMEM is freed once the last one issued is done
            if (issued > 0) barrier_wait(&ctl.empty[(issued - 1) % kStages], (issued - 1) / kStages & 1);
        }
    } else {
        // warps 2 to 17: a warp reaches the quarter of TMEM's rows that its number names modulo four
        const int quarter = warp & 3, group = (warp - 2) >> 2;
        float *bias = reinterpret_cast<float *>(extra) + (warp - 2) * kWarpColumns;
        int acc = 0, room_of = 0;
        uint32_t acc_parity = 0;
        bool ok = true;
        for (int item = first; item < items; item += step) {
            int split, tm, tn, kb0, kb1;
            a.tiles.at(static_cast<uint32_t>(item), split, tm, tn);
            range(split, kb0, kb1);
            if (kb0 == kb1) continue;
            const int m0 = tm * kTile + part * BM + quarter * 32, n0 = tn * kTile + group * kWarpColumns;  // below 2^31, see kMost
            const auto here = [&] { return tmem + acc * kTile + group * kWarpColumns + (static_cast<uint32_t>(quarter * 32) << 16); };
            uint32_t at = here();
            const auto arrived = [&] {  // once a wait has run out, nothing is waited for any more
                ok = ok && __all_sync(0xffffffffu, barrier_wait(&ctl.acc_full[acc], acc_parity));
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                return ok;
            };
            const auto release = [&] {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) barrier_arrive_at(first_blocks(smem_addr(&ctl.acc_empty[acc])));
            };
            const auto next = [&] {
                if (++acc == 2) acc = 0, acc_parity ^= 1;
                at = here();
            };
            // Pieces of a sum are added up in registers, and the whole goes back to where the last one lies.
            const auto ready = [&] {
                if constexpr (kInPieces<KIND>) {
                    if (a.k_blocks > a.pieces.first) {
                        float sum[kWarpColumns];
#pragma unroll
                        for (int i = 0; i < kWarpColumns; ++i) sum[i] = 0.f;
#pragma unroll 1
                        for (int left = a.k_blocks, piece = 0;; ++piece) {
                            if (!arrived()) return false;
#pragma unroll
                            for (int c = 0; c < kWarpColumns; c += 8) tmem_add8(at + c, sum + c);
                            left -= piece < 2 ? a.pieces.first : a.pieces.rest;
                            if (left <= 0) break;
                            release(), next();
                        }
#pragma unroll
                        for (int c = 0; c < kWarpColumns; c += 32) tmem_store32(at + c, sum + c);
                        tmem_stores_wait();
                        return true;
                    }
                }
                return arrived();
            };
            if (KIND == kStats || KIND == kLogits) {
                Sums mine;
                if constexpr (KIND == kLogits) mine = carry_logits<T, ENT>(a, at, m0 + lane, n0, bias, ready, release);
                else mine = carry_stats(a, at, m0 + lane, n0, bias, ready, release);
                // the four warps of these rows join their columns; two rooms, so that one barrier a tile is enough
                float *room = reinterpret_cast<float *>(extra + kBiasBytes) + ((room_of * 4 + quarter) * 4) * 96 + lane;
                room_of ^= 1;
                if (group > 0) room[group * 96] = mine.m, room[group * 96 + 32] = mine.s, room[group * 96 + 64] = mine.t;
                asm volatile("bar.sync %0, 128;" ::"r"(1 + quarter) : "memory");
                if (group == 0) {
                    Sums sums = mine;
#pragma unroll
                    for (int g = 1; g < 4; ++g) join(sums, {room[g * 96], room[g * 96 + 32], room[g * 96 + 64]}, a.c);
                    if (m0 < a.padded_rows) {
                        float *to = a.partial + static_cast<int64_t>(n0 / kTile) * 3 * a.padded_rows + m0 + lane;
                        to[0] = sums.m, to[a.padded_rows] = sums.s, to[2 * a.padded_rows] = sums.t;
                    }
                }
            } else if (KIND == kGrad) {
                carry_grad<T, ENT>(a, at, m0, n0, bias, ready, release);
            } else if (KIND == kHidden || KIND == kWeightParts) {
                carry_parts(a, at, split, m0, n0, ready, release);
            } else {
                carry_store<T>(a, at, m0, n0, extra + (warp - 2) * 1024, ready, release);
            }
            next();
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster.sync();  // no block leaves while its barriers are signalled or its operands read
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free<true>(tmem, 512);
    }
}

// A launch that may begin while the kernel before it ends; every kernel here starts with wait_for_previous().
template <class... P, class... A> int follow(void (*kernel)(P...), dim3 grid, int threads, int smem, int cluster, cudaStream_t s, A... args)
{
    cudaLaunchConfig_t config = {};
    config.gridDim = grid, config.blockDim = dim3(static_cast<unsigned>(threads));
    config.dynamicSmemBytes = static_cast<size_t>(smem);
    config.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster), attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    config.attrs = attr, config.numAttrs = cluster > 1 ? 2 : 1;
    SPDY_EVAL_TRY(cudaLaunchKernelEx(&config, kernel, static_cast<P>(args)...));
    return SPDY_OK;
}

// ---------------------------------------------------------------------------------------------- rows
struct RowArgs {
    int64_t R, V, padded_rows;
    int tiles;
    const float *partial, *token_logit;
    const void *tokens;
    int index_bits;
    float c, temperature;
    const float *in_lse, *in_entropy;          // a forward call's, when there is no partial
    float *logprob, *entropy, *lse;            // each may be NULL
    const float *grad_logprob, *grad_entropy;  // each may be NULL
    float *consts;                             // NULL without a gradient
};

// What carry_grad needs of a row, from the reference and base-2 logarithm of the sum relative to it.
// `x`: the token's logit, for the ones who use `known`.
__device__ __forceinline__ void write_consts(const RowArgs &a, int64_t r, int64_t token, float ref, float ls, float entropy, bool empty, float x)
{
    float ga = a.grad_logprob && token >= 0 ? a.grad_logprob[r] / a.temperature : 0.f;
    float gb = a.grad_entropy ? a.grad_entropy[r] / a.temperature : 0.f;
    if ((token >= a.V && a.grad_logprob) || ls != ls) ga = quiet_nan();  // the whole row's, its kept logits tell nothing
    if (empty) ref = ls = entropy = 0.f, ga = gb = 0.f;  // nothing allowed: no gradient
    float4 *to = reinterpret_cast<float4 *>(a.consts) + 2 * r;
    const float ab = ga + (a.grad_entropy ? gb * entropy : 0.f);
    to[0] = make_float4(ref, ls, ga, ab);
    const float y = min_nan(fmaf(x - ref, a.c, -ls), 0.f), known = ga - ex2(y) * fmaf(gb * kLn2, max_nan(y, -200.f), ab);
    to[1] = make_float4(gb * kLn2, __int_as_float(token < 0 || token >= a.V ? -1 : static_cast<int>(token)), known, 0.f);
}

// The largest bound on a row's gradient by its logits: |d| <= |ga| + |gb| (p |log p| + p H), p |log p| < 0.37, H <= log V.
__global__ void __launch_bounds__(256) scale_kernel(const RowArgs a, uint32_t *bits)
{
    wait_for_previous();
    float most = 0.f;
    const float spread = 0.37f + logf(static_cast<float>(a.V));
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; r < a.R; r += static_cast<int64_t>(gridDim.x) * 256) {
        const float ga = a.grad_logprob && token_at(a.tokens, a.index_bits, r) >= 0 ? fabsf(a.grad_logprob[r]) : 0.f, gb = a.grad_entropy ? fabsf(a.grad_entropy[r]) : 0.f;
        const float bound = (ga + gb * spread) / a.temperature;
        if (bound <= 3.4e38f) most = fmaxf(most, bound);
    }
    if (most > 0.f) atomicMax(bits, __float_as_uint(most));  // of whole numbers: the order does not matter
}

// What comes of a row's sums.
__device__ __forceinline__ void finish_row(const RowArgs &a, int64_t r, const Sums &sums)
{
    const int64_t token = a.tokens ? token_at(a.tokens, a.index_bits, r) : -1;
    const bool empty = sums.s == 0.f;
    const float log_s = logf(sums.s), entropy = empty ? 0.f : log_s - kLn2 * (sums.t / sums.s);
    if (a.lse) a.lse[r] = sums.m / a.temperature + log_s;
    if (a.entropy) a.entropy[r] = entropy;
    if (a.logprob) {
        float lp = 0.f;
        if (token >= a.V) lp = quiet_nan();
        else if (token >= 0) lp = empty ? neg_inf() : (a.token_logit[r] - sums.m) / a.temperature - log_s;
        a.logprob[r] = lp;
    }
    if (a.consts) write_consts(a, r, token, sums.m, log2f(sums.s), entropy, empty, a.token_logit && token >= 0 && token < a.V ? a.token_logit[r] : 0.f);
}

// Joins the tiles of 32 rows, a row to a lane: each warp every 32nd tile, eight of them at a time (their loads in flight together, one
// rescaling for all), then the warps.  2048 rows of 512 tiles: 34 us with a rescaling per tile and 16 warps, 10 this way.
constexpr int kRowWarps = 32, kRowTiles = 8;
__global__ void __launch_bounds__(32 * kRowWarps) rows_kernel(const RowArgs a)
{
    __shared__ float room[kRowWarps][3][32];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t r = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    // `N` sums at once; what is not there is the empty sum
    const auto join_all = [&](Sums &sums, const float *m, const float *s, const float *t, int count) {
        float top = sums.m;
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i)
            if (i < count) top = fmaxf(top, m[i]);
        raise(sums, top, a.c);
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i)
            if (i < count) {
                Sums one = {m[i], s[i], t[i]};
                raise(one, top, a.c);
                sums.s += one.s, sums.t += one.t;
            }
    };
    Sums sums = {neg_inf(), 0.f, 0.f};
    for (int tile = warp; tile < a.tiles; tile += kRowWarps * kRowTiles) {
        float m[kRowTiles], s[kRowTiles], t[kRowTiles];
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) {
            m[i] = neg_inf(), s[i] = t[i] = 0.f;
            if (tile + i * kRowWarps < a.tiles) {
                const float *from = a.partial + static_cast<int64_t>(tile + i * kRowWarps) * 3 * a.padded_rows + r;
                m[i] = from[0], s[i] = from[a.padded_rows], t[i] = from[2 * a.padded_rows];
            }
        }
        join_all(sums, m, s, t, kRowTiles);
    }
    room[warp][0][lane] = sums.m, room[warp][1][lane] = sums.s, room[warp][2][lane] = sums.t;
    __syncthreads();
    if (warp > 0 || r >= a.R) return;
    for (int w = 1; w < kRowWarps; w += kRowTiles) {
        float m[kRowTiles], s[kRowTiles], t[kRowTiles];
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) {
            m[i] = neg_inf(), s[i] = t[i] = 0.f;
            if (w + i < kRowWarps) m[i] = room[w + i][0][lane], s[i] = room[w + i][1][lane], t[i] = room[w + i][2][lane];
        }
        join_all(sums, m, s, t, kRowTiles);
    }
    finish_row(a, r, sums);
}

// The same for few rows, a block to a row, whose sums lie one behind the other.
__global__ void __launch_bounds__(256) few_rows_kernel(const RowArgs a)
{
    __shared__ float room[8][3];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float *from = a.partial + 3 * static_cast<int64_t>(blockIdx.x) * a.tiles;
    Sums sums = {neg_inf(), 0.f, 0.f};
#pragma unroll 4
    for (int i = threadIdx.x; i < a.tiles; i += 256) join(sums, {from[i], from[a.tiles + i], from[2 * a.tiles + i]}, a.c);
#pragma unroll
    for (int d = 16; d; d >>= 1) join(sums, {__shfl_xor_sync(0xffffffffu, sums.m, d), __shfl_xor_sync(0xffffffffu, sums.s, d), __shfl_xor_sync(0xffffffffu, sums.t, d)}, a.c);
    if (lane == 0) room[warp][0] = sums.m, room[warp][1] = sums.s, room[warp][2] = sums.t;
    __syncthreads();
    if (threadIdx.x > 0) return;
    for (int w = 1; w < 8; ++w) join(sums, {room[w][0], room[w][1], room[w][2]}, a.c);
    finish_row(a, blockIdx.x, sums);
}

// The same from a forward call's lse and entropy.
__global__ void __launch_bounds__(256) saved_rows_kernel(const RowArgs a)
{
    wait_for_previous();
    const int64_t r = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (r >= a.R) return;
    const float lse = a.in_lse[r];
    write_consts(a, r, a.tokens ? token_at(a.tokens, a.index_bits, r) : -1, lse * a.temperature, 0.f, a.in_entropy ? a.in_entropy[r] : 0.f, lse == neg_inf(), 0.f);
}

// ---------------------------------------------------------------------------------------------- few rows
// Logits of up to 4 rows: weight is streamed once by plain multiply-adds, four ids to a warp at a time, hidden comes from L1.  A block
// leaves one set of sums, as a tile does.  Bound by weight's bytes: 1 x 32768 x 768 12 us (the tensor cores 18), 1 x 131072 x 4096 186 (5.8 TB/s), 4 rows 217
// (212: from there on the tensor cores)
constexpr int kFewRows = 4, kFewIds = 4, kFewThreads = 256;
template <class T, int ROWS, bool WIDE>
__global__ void __launch_bounds__(kFewThreads) few_kernel(const T *hidden, int64_t ldh, const T *weight, int64_t ldw, int64_t R, int64_t V, int64_t D, float *logits,
                                                         int64_t ld_logits, const ProductArgs a)
{
    __shared__ float room[kFewThreads / 32][ROWS][3];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t warps = static_cast<int64_t>(gridDim.x) * (kFewThreads / 32);
    Sums sums[ROWS];
    int64_t token[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) sums[r] = {neg_inf(), 0.f, 0.f}, token[r] = r < R && a.token_logit ? token_at(a.tokens, a.index_bits, r) : -1;
    for (int64_t v0 = (static_cast<int64_t>(blockIdx.x) * (kFewThreads / 32) + warp) * kFewIds; v0 < V; v0 += warps * kFewIds) {
        float acc[ROWS][kFewIds];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int c = 0; c < kFewIds; ++c) acc[r][c] = 0.f;
        const T *w = weight + v0 * ldw;
        if (WIDE) {
#pragma unroll 3
            for (int64_t k = lane * 8; k < D; k += 256) {
                uint4 raw[kFewIds];
#pragma unroll
                for (int c = 0; c < kFewIds; ++c) raw[c] = v0 + c < V ? load_stream(w + c * ldw + k) : make_uint4(0, 0, 0, 0);
                float h[ROWS][8];
#pragma unroll
                for (int r = 0; r < ROWS; ++r) Elem<T>::unpack(r < R ? *reinterpret_cast<const uint4 *>(hidden + r * ldh + k) : make_uint4(0, 0, 0, 0), h[r]);
#pragma unroll
                for (int c = 0; c < kFewIds; ++c) {
                    float f[8];
                    Elem<T>::unpack(raw[c], f);
#pragma unroll
                    for (int r = 0; r < ROWS; ++r)
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[r][c] = fmaf(h[r][i], f[i], acc[r][c]);
                }
            }
        } else {
#pragma unroll 4
            for (int64_t k = lane; k < D; k += 32) {
                float f[kFewIds];
#pragma unroll
                for (int c = 0; c < kFewIds; ++c) f[c] = v0 + c < V ? Elem<T>::to_float(w[c * ldw + k]) : 0.f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const float h = r < R ? Elem<T>::to_float(hidden[r * ldh + k]) : 0.f;
#pragma unroll
                    for (int c = 0; c < kFewIds; ++c) acc[r][c] = fmaf(h, f[c], acc[r][c]);
                }
            }
        }
        const int64_t v = v0 + (lane & 3);  // the id whose logits this lane goes on with
        const float bias = a.bias && v < V ? value_at(a.bias, a.bias_type, v) : 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            // four sums over the lanes, of which each lane keeps one
            const bool up = lane & 1, high = lane & 2;
            float x = (up ? acc[r][1] : acc[r][0]) + __shfl_xor_sync(0xffffffffu, up ? acc[r][0] : acc[r][1], 1);
            const float y = (up ? acc[r][3] : acc[r][2]) + __shfl_xor_sync(0xffffffffu, up ? acc[r][2] : acc[r][3], 1);
            x = (high ? y : x) + __shfl_xor_sync(0xffffffffu, high ? x : y, 2);
#pragma unroll
            for (int d = 4; d < 32; d *= 2) x += __shfl_xor_sync(0xffffffffu, x, d);
            if (r >= R) continue;
            x = v < V ? x + bias : neg_inf();
            if (v == token[r] && lane < 4) a.token_logit[r] = x;
            if (logits && v < V && lane < 4) logits[r * ld_logits + v] = x;
            join(sums[r], {x, x == neg_inf() ? 0.f : 1.f, 0.f}, a.c);
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int d = 1; d < 4; d *= 2)
            join(sums[r], {__shfl_xor_sync(0xffffffffu, sums[r].m, d), __shfl_xor_sync(0xffffffffu, sums[r].s, d), __shfl_xor_sync(0xffffffffu, sums[r].t, d)}, a.c);
        if (lane == 0) room[warp][r][0] = sums[r].m, room[warp][r][1] = sums[r].s, room[warp][r][2] = sums[r].t;
    }
    __syncthreads();
    const int r = threadIdx.x;
    if (r >= ROWS || r >= R) return;
    Sums all = {neg_inf(), 0.f, 0.f};
    for (int q = 0; q < kFewThreads / 32; ++q) join(all, {room[q][r][0], room[q][r][1], room[q][r][2]}, a.c);
    float *to = a.partial + 3 * r * gridDim.x + blockIdx.x;
    to[0] = all.m, to[gridDim.x] = all.s, to[2 * gridDim.x] = all.t;
}

// The gradient by few rows' logits, in their place and in fp32 like them, and dbias; four columns to a thread.
template <bool ENT>
__global__ void __launch_bounds__(256) few_grad_kernel(float *logits, int64_t R, int64_t N, int64_t ld, const float *consts, float c, float *dbias)
{
    wait_for_previous();
    const int64_t n = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (n >= N) return;
    float sum[4] = {};
    for (int64_t r = 0; r < R; ++r) {
        const RowConsts k = row_consts(consts, r, 1.f);
        float4 *at = reinterpret_cast<float4 *>(logits + r * ld + n);  // ld is a multiple of 64
        float f[4] = {at->x, at->y, at->z, at->w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f[j] = grad_at<ENT>(fmaf(f[j] - k.ref, c, -k.ls), k);
            if (k.token == n + j) f[j] += k.hit;
            sum[j] += f[j];
        }
        *at = make_float4(f[0], f[1], f[2], f[3]);
    }
    if (dbias)
        for (int j = 0; j < 4 && n + j < N; ++j) dbias[n + j] = sum[j];
}

// dweight of few rows, and a block's share of dhidden, from the gradient in fp32 by plain multiply-adds: a block goes down a run of ids, a thread keeps
// PER columns (8, where all rows start on 16 bytes).  weight is read and dweight written once.
// Values and gradients, whole calls: 1 x 131072 x 4096 599 us (the tensor cores 796), 4 rows 628 (822); 4 x 32768 x 768 54 (67).
constexpr int kFewRun = 64;  // ids whose gradients lie in shared memory
template <class T, int ROWS, int PER>
__global__ void __launch_bounds__(256) few_products_kernel(const float *grad, int64_t ld, const T *hidden, int64_t ldh, const T *weight, int64_t ldw, int64_t R, int64_t V, int64_t D,
                                                           int64_t run, T *dweight, int64_t lddw, float *parts)
{
    __shared__ float g[ROWS][kFewRun];
    wait_for_previous();
    const int64_t d = (static_cast<int64_t>(blockIdx.y) * blockDim.x + threadIdx.x) * PER, first = blockIdx.x * run, end = min(first + run, V);
    const bool mine = d < D;
    float acc[ROWS][PER], h[ROWS][PER];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[r][i] = h[r][i] = 0.f;
        if (mine && r < R) {
            if constexpr (PER == 8) Elem<T>::unpack(*reinterpret_cast<const uint4 *>(hidden + r * ldh + d), h[r]);
            else h[r][0] = Elem<T>::to_float(hidden[r * ldh + d]);
        }
    }
    for (int64_t v0 = first; v0 < end; v0 += kFewRun) {
        const int count = static_cast<int>(min(end - v0, static_cast<int64_t>(kFewRun)));
        __syncthreads();
        for (int i = threadIdx.x; i < ROWS * kFewRun; i += blockDim.x) {
            const int r = i / kFewRun, v = i % kFewRun;
            g[r][v] = r < R && v < count ? grad[r * ld + v0 + v] : 0.f;
        }
        __syncthreads();
        if (!mine) continue;
        constexpr int U = 8;  // ids whose rows are on their way together (4 rows: 690 us with 4 of them, 628 with 8)
        for (int base = 0; base < count; base += U) {
            uint4 raw[U];
            float single[U];
            if (parts)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int64_t v = v0 + min(base + u, count - 1);
                    if constexpr (PER == 8) raw[u] = load_last(weight + v * ldw + d);
                    else single[u] = Elem<T>::to_float(weight[v * ldw + d]);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int v = base + u;
                if (v >= count) break;
                float w[PER], out[PER];
                if constexpr (PER == 8) Elem<T>::unpack(raw[u], w);
                else w[0] = single[u];
#pragma unroll
                for (int i = 0; i < PER; ++i) out[i] = 0.f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        if (parts) acc[r][i] = fmaf(g[r][v], w[i], acc[r][i]);
                        out[i] = fmaf(g[r][v], h[r][i], out[i]);
                    }
                if (dweight) {
                    T *to = dweight + (v0 + v) * lddw + d;
                    if constexpr (PER == 8) store_last(to, Elem<T>::pack(out));
                    else *to = Elem<T>::from_float(out[0]);
                }
            }
        }
    }
    if (!parts || !mine) return;
    for (int r = 0; r < ROWS && r < R; ++r)
#pragma unroll
        for (int i = 0; i < PER; ++i) parts[(static_cast<int64_t>(blockIdx.x) * R + r) * D + d + i] = acc[r][i];
}

// dhidden of few rows: the blocks' shares in a fixed order, eight runs of them to a column.
template <class T> __global__ void __launch_bounds__(256) few_finish_kernel(const float *parts, int blocks, int64_t R, int64_t D, T *dhidden, int64_t lddh)
{
    __shared__ float room[8][32];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t d = static_cast<int64_t>(blockIdx.x) * 32 + lane, r = blockIdx.y;
    float sum = 0.f;
    if (d < D)
#pragma unroll 8
        for (int b = warp; b < blocks; b += 8) sum += parts[(b * R + r) * D + d];
    room[warp][lane] = sum;
    __syncthreads();
    if (warp > 0 || d >= D) return;
    for (int w = 1; w < 8; ++w) sum += room[w][lane];
    dhidden[r * lddh + d] = Elem<T>::from_float(sum);
}

// ---------------------------------------------------------------------------------------------- gradient by kept logits
// Codes into the gradient, in place: eight columns to a thread, eight rows at a time; FINE: of 32 rows, which it adds up for dbias.
// Memory bound: 2 bytes in (3), 2 out; 4096 x 32768 97 us (5.5 TB/s).  Blocks of 128, of which small calls have enough (with 256
// threads 512 x 30001 x 768, the whole call, took 9 us longer).
constexpr int kGradRows = 8, kGradThreads = 128;
template <bool FINE> constexpr int kGradBlock = FINE ? 32 : kGradRows;
template <class T, bool ENT, bool FINE>
__global__ void __launch_bounds__(kGradThreads) grad_kernel(uint16_t *codes, const uint8_t *fine, const float *tops, int64_t padded_rows, int64_t M, int64_t N, int64_t ld, const float *consts,
                                                   float c, const uint32_t *scale_bits, float *column_sums, int64_t low)
{
    __shared__ RowConsts rows[kGradBlock<FINE>];
    wait_for_previous();
    const int64_t n = (static_cast<int64_t>(blockIdx.x) * kGradThreads + threadIdx.x) * 8;
    for (int64_t m0 = static_cast<int64_t>(blockIdx.y) * kGradBlock<FINE>; m0 < max(M, low); m0 += static_cast<int64_t>(gridDim.y) * kGradBlock<FINE>) {
        const int count = static_cast<int>(max(min(M - m0, static_cast<int64_t>(kGradBlock<FINE>)), static_cast<int64_t>(0)));
        __syncthreads();
        if (threadIdx.x < count) rows[threadIdx.x] = row_consts(consts, m0 + threadIdx.x, power_of_two(scale_power(scale_bits)));
        __syncthreads();
        if (n >= N) continue;
        float sum[8] = {};
#pragma unroll 1
        for (int first = 0; first < count; first += kGradRows) {
            uint4 raw[kGradRows];
            uint2 bits[kGradRows];
            float top[kGradRows];
#pragma unroll
            for (int i = 0; i < kGradRows; ++i)
                if (first + i < count) {  // ld is a multiple of 64: columns behind N are there, and nobody reads what becomes of them
                    const int64_t m = m0 + first + i;
                    raw[i] = load_last(codes + m * ld + n);
                    if (FINE) bits[i] = *reinterpret_cast<const uint2 *>(fine + m * ld + n);
                    top[i] = tops[n / kCodes * padded_rows + m];
                }
#pragma unroll
            for (int i = 0; i < kGradRows; ++i) {
                if (first + i >= count) break;
                const RowConsts k = rows[first + i];
                const float base = fmaf(top[i] - k.ref, c, -k.ls);
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t high = j % 2 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
                    const uint32_t code = FINE ? high << 7 | __byte_perm(j < 4 ? bits[i].x : bits[i].y, 0, 0x4440 | j % 4) : high;
                    const float steps = __uint_as_float(0x4b000000u | code) - 8388608.f;
                    f[j] = grad_at<ENT>(high == kNothing ? neg_inf() : fmaf(steps, -1.f / kCodeSteps<T, FINE>, base), k);
                }
                const int64_t at = k.token - n;
                if (at >= 0 && at < 8)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (at == j) f[j] = k.known;
                if (FINE)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] += f[j];
                const uint4 rounded = Elem<T>::pack(f);
                *reinterpret_cast<uint4 *>(codes + (m0 + first + i) * ld + n) = rounded;
                if (low) *reinterpret_cast<uint4 *>(codes + (low + m0 + first + i) * ld + n) = lower_halves<T>(f, rounded);
            }
        }
        for (int64_t m = m0 + count; m < low && m < m0 + kGradBlock<FINE>; ++m) *reinterpret_cast<uint4 *>(codes + m * ld + n) = make_uint4(0, 0, 0, 0);
        if (FINE && count > 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) column_sums[m0 / 32 * ld + n + j] = sum[j];
    }
}

// ---------------------------------------------------------------------------------------------- sums of parts
// out[m][n] = sum over the splits of parts[split][m][n] (and, with `low`, of parts[split][low + m][n]), in their order, times 2^-scale, rounded once; eight
// columns to a thread; `rows`: of a part.
// `wide`: every row of out starts on 16 bytes.  Index: 32 bits where they are enough (a division by a 64-bit number cost more than all the rest).
template <class T, class Index>
__global__ void __launch_bounds__(256) finish_kernel(const float *parts, int splits, int64_t rows, int64_t low, int64_t M, int64_t N, int64_t ldp, const uint32_t *scale_bits, T *out, int64_t ldo,
                                                     int wide)
{
    wait_for_previous();
    const float scale = power_of_two(-scale_power(scale_bits));
    const Index across = static_cast<Index>(ldp / 8), total = static_cast<Index>(M) * across;
    for (Index i = static_cast<Index>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<Index>(gridDim.x) * 256) {
        const Index row = i / across;
        const int64_t m = row, n = static_cast<int64_t>(i - row * across) * 8;
        float sum[8] = {};
        for (int half = 0; half < (low ? 2 : 1); ++half)
#pragma unroll 2
            for (int s = 0; s < splits; ++s) {
                uint4 lo, hi;
                load32(parts + (s * rows + half * low + m) * ldp + n, lo, hi);
                float f[8];
                Elem<float>::unpack(lo, f), Elem<float>::unpack(hi, f + 4);
#pragma unroll
                for (int k = 0; k < 8; ++k) sum[k] += f[k];
            }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum[k] *= scale;
        T *to = out + m * ldo + n;
        if (wide && n + 8 <= N) {
            *reinterpret_cast<uint4 *>(to) = Elem<T>::pack(sum);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (n + k < N) to[k] = Elem<T>::from_float(sum[k]);
        }
    }
}
template <class T> int finish(const float *parts, int splits, int64_t rows, int64_t low, int64_t M, int64_t N, int64_t ldp, const uint32_t *scale_bits, T *out, int64_t ldo, cudaStream_t s)
{
    const int wide = aligned(out, 16) && ldo % 8 == 0;
    const int64_t total = M * (ldp / 8), most = static_cast<int64_t>(sm_count()) * 8, want = (total + 255) / 256;
    const unsigned blocks = static_cast<unsigned>(want < most ? want : most);
    if (total + most * 256 < (1ll << 32)) return follow(finish_kernel<T, uint32_t>, dim3(blocks), 256, 0, 1, s, parts, splits, rows, low, M, N, ldp, scale_bits, out, ldo, wide);
    return follow(finish_kernel<T, uint64_t>, dim3(blocks), 256, 0, 1, s, parts, splits, rows, low, M, N, ldp, scale_bits, out, ldo, wide);
}

// dbias of a piece: the row groups' sums in their order, eight runs of them to a column.
__global__ void __launch_bounds__(256) bias_kernel(const float *sums, int64_t groups, int64_t N, int64_t ld, const uint32_t *scale_bits, float *dbias, int add)
{
    __shared__ float room[8][32];
    wait_for_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    float sum = 0.f;
    if (n < N)
        for (int64_t g = warp; g < groups; g += 8) sum += sums[g * ld + n];
    room[warp][lane] = sum;
    __syncthreads();
    if (warp > 0 || n >= N) return;
    for (int w = 1; w < 8; ++w) sum += room[w][lane];
    sum *= power_of_two(-scale_power(scale_bits));
    dbias[n] = add ? dbias[n] + sum : sum;
}

// ---------------------------------------------------------------------------------------------- launches
int64_t div_up(int64_t x, int64_t y) { return (x + y - 1) / y; }
size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// By ids: the gradient by the logits is kept for as many ids at a time as this much memory holds, 2048 at least.
constexpr int64_t kPieceBytes = 256ll << 20, kLeastPiece = 2048;
// By rows: the logits, for as many rows as this much memory holds; not where that is few, since dweight's fp32 sums are read and
// written for each.  8192 rows (bf16, ms by rows and by ids): room for 2048 (131072 ids, width 1024) 6.8, 6.5; for 1766 (151936) 9.0, 7.7, at 4096 30.1,
// 31.1; for 1342 (200000) 12.3, 10.4, at 4096 41.2, 42.4; with dbias for 1365 (131072) 9.6, 8.3, for 1178 (151936) at 4096 33.6, 31.8.
constexpr int64_t kLogitBytes = 512ll << 20, kLeastRows = 2048;

// Whether keeping the logits costs less than multiplying them again, which the width decides.  4096 x 32768 bf16, us by rows and by ids: width 512 486,
// 488, 768 700, 701, 1024 828, 844; with dbias (another byte per logit) 640 778, 700, 768 840, 771, 1024 980, 968.  Fewer logits stay in L2 in part:
// 1021 x 50001 with dbias 768 283, 333, 1024 405, 429; 512 x 30001 with dbias 512 115, 118, 768 128, 129, without 256 95, 98.
bool keeps_logits(int64_t R, int64_t V, int64_t D, bool bias) { return D >= (bias && R > (1ll << 26) / V ? 1024 : 512); }

// Sums of a row's tiles, 12 bytes each, for as many rows at a time as this much memory holds, 4096 at least.
constexpr int64_t kPartialBytes = 32ll << 20, kLeastStats = 4096;

struct Layout {
    size_t hidden, weight, partial, token_logit, consts, scale, logits, tops, fine, piece, parts, weight_sums, sums, total;
    int64_t padded_rows, rows, stat_rows, width, ld_piece, ld_parts;  // rows, width: what is worked on at a time; stat_rows: for values
    int64_t low, piece_rows;  // of the piece: where the lower halves of g begin (0: it has none), all of them
    int hidden_splits, weight_splits;
    bool by_rows;
};

// How many parts the sum of a product of few tiles is split into, so that it fills the pairs of multiprocessors: the least estimated time in stages
// (0.55 us each), a part costing its share, about five more for its way in and out, and the memory traffic of its M x N fp32 sums.
int choose_splits(int64_t M, int64_t N, int64_t k_blocks)
{
    const int64_t pairs = sm_count() / 2, tiles = div_up(M, kTile) * div_up(N, kTile);
    const double traffic = static_cast<double>(M) * static_cast<double>(N) * 2.2e-6;
    int best = 1;
    double least = 1e300;
    for (int s = 1; s <= 64 && s <= k_blocks; ++s) {
        const double time = static_cast<double>(div_up(tiles * s, pairs)) * (static_cast<double>(div_up(k_blocks, s)) + 5.0) + traffic * s;
        if (time < least) least = time, best = s;
    }
    return best;
}

// Copies of operands get rows of whole 128 bytes: TMA's boxes then touch no line twice (1021 x 50001 x 1000: 108 us with rows of 2000 bytes,
// 84 us with 2048).
int64_t copy_ld(int64_t D) { return div_up(D, 64) * 64; }
size_t copy_bytes(int64_t rows, int64_t D) { return static_cast<size_t>(rows) * static_cast<size_t>(copy_ld(D)) * 2; }

// Few rows need no tensor cores.  (Nor are fp32's digits then given away: with one row whose token is all but certain the gradient is the
// small difference 1 - p.)
bool is_few(int64_t R) { return R <= kFewRows; }
// The gradient of few rows goes into the products in two halves of 16 bits, the second one what rounding took from the first: with few numbers to a sum the
// rounding of one, up to 2^-9, shows (half precision, 5 to 44 rows: dhidden and dweight were off by up to 1.6 times the last rounding alone; with more rows
// by 1.4 times).  The halves lie below one another, at most 128 rows: one tile of dhidden's product and one stage of dweight's.  Whole calls take 1 to 18 % longer
// (33 x 32768 x 768 64 -> 71 us, 33 x 131072 x 4096 737 -> 741; with 128 rows it would be 7 to 26 %).
constexpr int64_t kHalvesRows = 64;
int64_t few_blocks() { return static_cast<int64_t>(sm_count()) * 4; }

Layout lay_out(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int64_t R, int64_t V, int64_t D, bool stats, bool grads, bool bias)
{
    Layout l = {};
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += rounded(bytes);
        return here;
    };
    l.rows = R, l.width = V;
    if (is_few(R)) {
        l.partial = take(static_cast<size_t>(few_blocks()) * 3 * R * 4);
        l.token_logit = take(static_cast<size_t>(R) * 4);
        if (grads) {
            l.ld_piece = div_up(V, 64) * 64;
            l.consts = take(static_cast<size_t>(R) * kConsts * 4);
            l.logits = take(static_cast<size_t>(R) * l.ld_piece * 4);
            l.parts = take(static_cast<size_t>(few_blocks()) * R * D * 4);
        }
        l.total = at;
        return l;
    }
    l.hidden = take(tma_ok(hidden, ldh) ? 0 : copy_bytes(R, D));
    l.weight = take(tma_ok(weight, ldw) ? 0 : copy_bytes(V, D));
    if (grads) {
        l.ld_piece = div_up(V, 64) * 64;
        l.low = R <= kHalvesRows ? div_up(R, BK) * BK : 0;
        const int64_t most = kLogitBytes / (bias ? 3 : 2) / l.ld_piece;  // rows
        l.by_rows = stats && keeps_logits(R, V, D, bias) && (R + l.low <= most || most >= kLeastRows);
        if (l.by_rows) {
            const int64_t pieces = R <= most ? 1 : div_up(R, most / kTile * kTile);
            if (pieces > 1) l.rows = div_up(div_up(R, pieces), kTile) * kTile;  // of one size
        } else {
            int64_t width = kPieceBytes / 2 / (R + l.low) / kTile * kTile;
            if (width < kLeastPiece) width = kLeastPiece;
            const int64_t pieces = div_up(V, width);
            width = div_up(div_up(V, pieces), kTile) * kTile;
            if (width < V) l.width = l.ld_piece = width;
        }
        const bool once = l.rows == R;
        l.ld_parts = div_up(D, 8) * 8;
        l.piece_rows = l.low + l.rows;
        l.hidden_splits = choose_splits(l.piece_rows, D, div_up(l.width, kStageK));
        l.weight_splits = once ? choose_splits(l.width, D, div_up(l.piece_rows, kStageK)) : 1;
        l.consts = take(static_cast<size_t>(l.rows) * kConsts * 4);
        l.scale = take(256);
        if (l.by_rows) l.tops = take(static_cast<size_t>(l.ld_piece / kCodes) * (div_up(l.rows, 32) * 32) * 4);
        l.piece = take(static_cast<size_t>(l.piece_rows) * l.ld_piece * 2);
        l.parts = take(static_cast<size_t>(l.hidden_splits) * l.piece_rows * l.ld_parts * 4);
        if (!once || l.weight_splits > 1) l.weight_sums = take(static_cast<size_t>(l.weight_splits) * l.width * l.ld_parts * 4);
        if (l.by_rows && bias) l.fine = take(static_cast<size_t>(l.rows) * l.ld_piece);
        if (bias) l.sums = take(static_cast<size_t>(div_up(l.rows, 32)) * l.ld_piece * 4);
    }
    l.stat_rows = l.rows;
    if (stats) {
        if (!l.by_rows) {
            const int64_t most = kPartialBytes / 12 / div_up(V, kTile) / kTile * kTile, rows = most > kLeastStats ? most : kLeastStats;
            if (rows < R) l.stat_rows = div_up(div_up(R, div_up(R, rows)), kTile) * kTile;  // of one size
        }
        l.padded_rows = div_up(l.stat_rows, 32) * 32;
        l.partial = take(static_cast<size_t>(div_up(V, kTile)) * 3 * l.padded_rows * 4);
        l.token_logit = take(static_cast<size_t>(l.stat_rows) * 4);
    }
    l.total = at;
    return l;
}

struct HeadArgs {
    const void *hidden, *weight, *bias, *tokens;
    int64_t ldh, ldw, R, V, D;
    int dtype, bias_type, index_bits;
    float temperature;
    const float *in_lse, *in_entropy, *grad_logprob, *grad_entropy;
    float *logprob, *entropy, *lse;
    void *dhidden, *dweight;
    int64_t lddh, lddw;
    float *dbias;
    bool stats, grads;
};

// A map of a row-major matrix [rows][columns], boxes of 64 columns and `box_rows` rows.
int map_of(CUtensorMap *map, const void *p, int64_t ld, int64_t rows, int64_t columns, int dtype, int box_rows) { return make_map(map, p, ld, rows, columns, dtype, box_rows); }

template <class T, int KIND, bool ENT> int launch_product(const CUtensorMap &ma, const CUtensorMap &mb, ProductArgs a, int64_t K, int group, int splits, cudaStream_t s)
{
    const int64_t tm = div_up(a.M, kTile), tn = div_up(a.N, kTile);
    if (tm * tn * splits > 0x3fffffff) return SPDY_ERR_UNSUPPORTED;
    a.tiles = Tiles(static_cast<int>(tm), static_cast<int>(tn), group), a.splits = splits, a.per_split = Divisor(static_cast<uint32_t>(splits));
    a.k_blocks = static_cast<int>(div_up(K, kStageK));
    if (a.wrap == 0) a.wrap = INT_MAX;
    const int items = static_cast<int>(tm * tn) * splits, pairs = sm_count() / 2;
    auto *kernel = product_kernel<T, KIND, ENT>;
    SPDY_EVAL_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<KIND>()));
    return follow(kernel, dim3(static_cast<unsigned>((items < pairs ? items : pairs) * 2)), kThreads, smem_bytes<KIND>(), 2, s, ma, mb, a);
}

// Tiles down that are worked on side by side: in a product over the width, as many as leave their rows of hidden (or of the piece) in L2.
int group_of(int64_t K)
{
    const int64_t g = (48ll << 20) / (kTile * K * 2);
    return static_cast<int>(g < 8 ? 8 : g > 4096 ? 4096 : g);
}

#define HEAD_TRY(expr)                     \
    do {                                   \
        const int rc__ = (expr);           \
        if (rc__ != SPDY_OK) return rc__;  \
    } while (0)

// The steps of a call on some rows (from r0) and ids (from v0).
template <class T> struct Head {
    const HeadArgs &h;
    const Layout &l;
    char *ws;
    cudaStream_t s;
    ProductArgs base;
    CUtensorMap hidden, weight, hidden_columns, weight_columns;

    float *floats(size_t at) const { return reinterpret_cast<float *>(ws + at); }

    // All of few rows.
    template <int ROWS> int few(RowArgs rows)
    {
        ProductArgs a = base;
        a.partial = floats(l.partial), a.token_logit = rows.tokens ? floats(l.token_logit) : nullptr;
        const int64_t want = div_up(h.V, kFewIds * (kFewThreads / 32)), most = few_blocks();
        const unsigned blocks = static_cast<unsigned>(want < most ? want : most);
        const T *x = static_cast<const T *>(h.hidden), *w = static_cast<const T *>(h.weight);
        const bool wide = tma_ok(x, h.ldh) && tma_ok(w, h.ldw) && h.D % 8 == 0;
        float *logits = h.grads ? floats(l.logits) : nullptr;
        HEAD_TRY(follow(wide ? few_kernel<T, ROWS, true> : few_kernel<T, ROWS, false>, dim3(blocks), kFewThreads, 0, 1, s, x, h.ldh, w, h.ldw, h.R, h.V, h.D, logits, l.ld_piece, a));
        if (h.stats) {
            rows.partial = a.partial, rows.token_logit = a.token_logit, rows.tiles = static_cast<int>(blocks);
            HEAD_TRY(follow(few_rows_kernel, dim3(static_cast<unsigned>(h.R)), 256, 0, 1, s, rows));
        } else {
            HEAD_TRY(follow(saved_rows_kernel, dim3(1), 256, 0, 1, s, rows));
        }
        if (!h.grads) return SPDY_OK;
        HEAD_TRY(follow(h.grad_entropy ? few_grad_kernel<true> : few_grad_kernel<false>, dim3(static_cast<unsigned>(div_up(h.V, 1024))), 256, 0, 1, s, logits, h.R, h.V, l.ld_piece,
                        base.consts, base.c, h.dbias));
        if (!h.dhidden && !h.dweight) return SPDY_OK;
        T *dweight = static_cast<T *>(h.dweight);
        const bool wide_too = wide && (!dweight || tma_ok(dweight, h.lddw));
        const int64_t columns = div_up(h.D, wide_too ? 8 : 1), threads = columns < 256 ? div_up(columns, 32) * 32 : 256, across = div_up(columns, threads);
        const int64_t down = most / across > 1 ? most / across : 1, run = div_up(div_up(h.V, down), 8) * 8;
        const unsigned runs = static_cast<unsigned>(div_up(h.V, run));
        if (across > 65535) return SPDY_ERR_UNSUPPORTED;
        float *parts = h.dhidden ? floats(l.parts) : nullptr;
        HEAD_TRY(follow(wide_too ? few_products_kernel<T, ROWS, 8> : few_products_kernel<T, ROWS, 1>, dim3(runs, static_cast<unsigned>(across)), static_cast<int>(threads), 0, 1, s,
                        logits, l.ld_piece, x, h.ldh, w, h.ldw, h.R, h.V, h.D, run, dweight, h.lddw, parts));
        if (!h.dhidden) return SPDY_OK;
        return follow(few_finish_kernel<T>, dim3(static_cast<unsigned>(div_up(h.D, 32)), static_cast<unsigned>(h.R)), 256, 0, 1, s, parts, static_cast<int>(runs), h.R, h.D,
                      static_cast<T *>(h.dhidden), h.lddh);
    }

    // Sums of rows' exponentials and what comes of them; KIND kLogits keeps the logits.
    template <int KIND> int stats(RowArgs rows, int64_t r0)
    {
        ProductArgs a = base;
        a.M = rows.R, a.N = h.V, a.a_row0 = static_cast<int>(r0);
        a.tokens = rows.tokens;
        a.partial = floats(l.partial), a.token_logit = rows.tokens ? floats(l.token_logit) : nullptr;
        if (KIND == kLogits) a.out = ws + l.piece, a.ldo = l.ld_piece, a.tops = floats(l.tops), a.fine = h.dbias ? reinterpret_cast<uint8_t *>(ws + l.fine) : nullptr;
        if (KIND == kLogits && h.dbias) HEAD_TRY((launch_product<T, KIND, true>(hidden, weight, a, h.D, group_of(h.D), 1, s)));
        else HEAD_TRY((launch_product<T, KIND, false>(hidden, weight, a, h.D, group_of(h.D), 1, s)));
        rows.partial = a.partial, rows.token_logit = a.token_logit, rows.tiles = static_cast<int>(div_up(h.V, kTile));
        return follow(rows_kernel, dim3(static_cast<unsigned>(div_up(rows.R, 32))), 32 * kRowWarps, 0, 1, s, rows);
    }
    // The gradient by the kept logits of m rows (from r0), and dbias.
    int gradient(int64_t m, int64_t r0)
    {
        const bool fine = h.dbias != nullptr;
        const int64_t down = div_up(m > l.low ? m : l.low, fine ? kGradBlock<true> : kGradBlock<false>);
        const dim3 grid(static_cast<unsigned>(div_up(h.V, kGradThreads * 8)), static_cast<unsigned>(down < 65535 ? down : 65535));
        uint16_t *codes = reinterpret_cast<uint16_t *>(ws + l.piece);
        const uint8_t *low = reinterpret_cast<const uint8_t *>(ws + l.fine);
        auto *kernel = fine ? (h.grad_entropy ? grad_kernel<T, true, true> : grad_kernel<T, false, true>) : h.grad_entropy ? grad_kernel<T, true, false> : grad_kernel<T, false, false>;
        HEAD_TRY(follow(kernel, grid, kGradThreads, 0, 1, s, codes, low, floats(l.tops), l.padded_rows, m, h.V, l.ld_piece, base.consts, base.c, base.scale_bits, floats(l.sums),
                        l.low));
        return fine ? finish_bias(m, h.V, 0, r0 > 0) : SPDY_OK;
    }
    // The gradient by the logits of all rows and ids v0 .. v0 + n - 1, which are multiplied again; dbias of these ids.
    int gradient_again(int64_t n, int64_t v0)
    {
        ProductArgs a = base;
        a.M = h.R, a.N = n, a.v0 = v0, a.b_row0 = static_cast<int>(v0);
        a.out = ws + l.piece, a.ldo = l.ld_piece, a.low = static_cast<int>(l.low), a.below = l.low * l.ld_piece * 2;
        if (h.dbias) a.column_sums = floats(l.sums), a.ld_sums = l.ld_piece;
        else a.pieces = kGradPieces;  // g in 16 bits shows nothing of it
        if (h.grad_entropy) HEAD_TRY((launch_product<T, kGrad, true>(hidden, weight, a, h.D, group_of(h.D), 1, s)));
        else HEAD_TRY((launch_product<T, kGrad, false>(hidden, weight, a, h.D, group_of(h.D), 1, s)));
        return h.dbias ? finish_bias(h.R, n, v0, false) : SPDY_OK;
    }
    int finish_bias(int64_t m, int64_t n, int64_t v0, bool add)
    {
        return follow(bias_kernel, dim3(static_cast<unsigned>(div_up(n, 32))), 256, 0, 1, s, floats(l.sums), div_up(m, 32), n, l.ld_piece, base.scale_bits, h.dbias + v0, add);
    }
    // dhidden's sums and dweight from the gradient of m rows (from r0) and n ids (from v0), added to what earlier rows or ids gave.
    int products(int64_t m, int64_t r0, int64_t n, int64_t v0)
    {
        const int64_t rows = l.low + m;  // of the piece
        CUtensorMap piece;
        if (h.dhidden) {
            HEAD_TRY(map_of(&piece, ws + l.piece, l.ld_piece, rows, n, h.dtype, BM));
            ProductArgs b = {};
            b.M = rows, b.N = h.D, b.b_row0 = static_cast<int>(v0), b.out = floats(l.parts), b.ldo = l.ld_parts, b.add = v0 > 0;
            HEAD_TRY((launch_product<T, kHidden, false>(piece, weight_columns, b, n, 8, l.hidden_splits, s)));
        }
        if (!h.dweight) return SPDY_OK;
        HEAD_TRY(map_of(&piece, ws + l.piece, l.ld_piece, rows, n, h.dtype, BK));
        T *out = static_cast<T *>(h.dweight) + v0 * h.lddw;
        ProductArgs b = {};
        b.M = n, b.N = h.D, b.b_row0 = static_cast<int>(r0), b.wrap = static_cast<int>(l.low);
        const bool last = r0 + m == h.R;
        if (l.weight_splits > 1 || !last) {
            b.out = floats(l.weight_sums), b.ldo = l.ld_parts, b.add = r0 > 0;
            HEAD_TRY((launch_product<T, kWeightParts, false>(piece, hidden_columns, b, rows, 8, l.weight_splits, s)));
            return last ? finish<T>(floats(l.weight_sums), l.weight_splits, n, 0, n, h.D, l.ld_parts, base.scale_bits, out, h.lddw, s) : SPDY_OK;
        }
        b.out = out, b.ldo = h.lddw, b.scale_bits = base.scale_bits;
        b.width = aligned(out, 32) && h.lddw % 16 == 0 ? 32 : aligned(out, 16) && h.lddw % 8 == 0 ? 16 : 0;
        if (r0 > 0) b.sums = floats(l.weight_sums), b.ld_old = l.ld_parts;
        return launch_product<T, kWeight, false>(piece, hidden_columns, b, rows, 8, 1, s);
    }
    int finish_hidden(int64_t m, int64_t r0)
    {
        return finish<T>(floats(l.parts), l.hidden_splits, l.low + m, l.low, m, h.D, l.ld_parts, base.scale_bits, static_cast<T *>(h.dhidden) + r0 * h.lddh, h.lddh, s);
    }
};

template <class T> int run_head(HeadArgs h, void *workspace, cudaStream_t s)
{
    const Layout l = lay_out(h.hidden, h.ldh, h.weight, h.ldw, h.R, h.V, h.D, h.stats, h.grads, h.dbias != nullptr);
    char *ws = static_cast<char *>(workspace);
    const int64_t R = h.R, V = h.V, D = h.D;
    const bool few = is_few(R);
    Repack p = {};
    p.K = D, p.ldto = copy_ld(D);
    if (!few && !tma_ok(h.hidden, h.ldh)) {
        p.from[0] = static_cast<const uint16_t *>(h.hidden), p.ld[0] = h.ldh, p.rows[0] = R, p.to[0] = reinterpret_cast<uint16_t *>(ws + l.hidden);
        h.hidden = ws + l.hidden, h.ldh = p.ldto;
    }
    if (!few && !tma_ok(h.weight, h.ldw)) {
        p.from[1] = static_cast<const uint16_t *>(h.weight), p.ld[1] = h.ldw, p.rows[1] = V, p.to[1] = reinterpret_cast<uint16_t *>(ws + l.weight);
        h.weight = ws + l.weight, h.ldw = p.ldto;
    }
    HEAD_TRY(repack(p, s));
    CUtensorMap hidden = {}, weight = {};
    if (!few) {
        HEAD_TRY(map_of(&hidden, h.hidden, h.ldh, R, D, h.dtype, BM));
        HEAD_TRY(map_of(&weight, h.weight, h.ldw, V, D, h.dtype, BM));
    }

    RowArgs rows = {};
    rows.R = R, rows.V = V, rows.padded_rows = l.padded_rows;
    rows.tokens = h.tokens, rows.index_bits = h.index_bits, rows.c = kLog2e / h.temperature, rows.temperature = h.temperature;
    rows.in_lse = h.in_lse, rows.in_entropy = h.in_entropy, rows.logprob = h.logprob, rows.entropy = h.entropy, rows.lse = h.lse;
    rows.grad_logprob = h.grad_logprob, rows.grad_entropy = h.grad_entropy;
    ProductArgs base = {};
    base.bias = h.bias, base.bias_type = h.bias_type, base.tokens = h.tokens, base.index_bits = h.index_bits;
    base.c = rows.c, base.pieces = kLogitPieces, base.padded_rows = l.padded_rows;
    if (h.grads) {
        rows.consts = reinterpret_cast<float *>(ws + l.consts);
        if (!few && h.dtype == SPDY_F16) {
            uint32_t *bits = reinterpret_cast<uint32_t *>(ws + l.scale);
            SPDY_EVAL_TRY(cudaMemsetAsync(bits, 0, 4, s));
            const int64_t blocks = div_up(R, 256), most = sm_count();
            HEAD_TRY(follow(scale_kernel, dim3(static_cast<unsigned>(blocks < most ? blocks : most)), 256, 0, 1, s, rows, bits));
            base.scale_bits = bits;
        }
        base.consts = rows.consts;
    }
    Head<T> g = {h, l, ws, s, base, hidden, weight, {}, {}};
    if (few) return R == 1 ? g.template few<1>(rows) : R == 2 ? g.template few<2>(rows) : g.template few<4>(rows);
    if (h.grads) {
        HEAD_TRY(map_of(&g.hidden_columns, h.hidden, h.ldh, R, D, h.dtype, BK));
        HEAD_TRY(map_of(&g.weight_columns, h.weight, h.ldw, V, D, h.dtype, BK));
    }
    const auto part = [&](int64_t r0, int64_t n) {  // the same of rows r0 .. r0 + n - 1
        RowArgs some = rows;
        some.R = n;
        if (some.tokens) some.tokens = static_cast<const char *>(rows.tokens) + r0 * static_cast<int64_t>(h.index_bits / 8);
        for (float **p : {&some.logprob, &some.entropy, &some.lse}) *p = *p ? *p + r0 : nullptr;
        for (const float **p : {&some.grad_logprob, &some.grad_entropy}) *p = *p ? *p + r0 : nullptr;
        return some;
    };
    if (h.grads && l.by_rows) {
        for (int64_t r0 = 0; r0 < R; r0 += l.rows) {
            const int64_t n = R - r0 < l.rows ? R - r0 : l.rows;
            HEAD_TRY(g.template stats<kLogits>(part(r0, n), r0));
            HEAD_TRY(g.gradient(n, r0));
            HEAD_TRY(g.products(n, r0, V, 0));
            if (h.dhidden) HEAD_TRY(g.finish_hidden(n, r0));
        }
    } else {
        if (h.stats) {
            for (int64_t r0 = 0; r0 < R; r0 += l.stat_rows) {
                RowArgs some = part(r0, R - r0 < l.stat_rows ? R - r0 : l.stat_rows);
                if (some.consts) some.consts += r0 * kConsts;
                HEAD_TRY(g.template stats<kStats>(some, r0));
            }
        } else {
            HEAD_TRY(follow(saved_rows_kernel, dim3(static_cast<unsigned>(div_up(R, 256))), 256, 0, 1, s, rows));
        }
        if (!h.grads) return SPDY_OK;
        for (int64_t v0 = 0; v0 < V; v0 += l.width) {
            const int64_t n = V - v0 < l.width ? V - v0 : l.width;
            HEAD_TRY(g.gradient_again(n, v0));
            HEAD_TRY(g.products(R, 0, n, v0));
        }
        if (h.dhidden) HEAD_TRY(g.finish_hidden(R, 0));
    }
    return SPDY_OK;
}

constexpr int64_t kMost = 0x7fff0000;  // rows, ids, width: tile coordinates are 32-bit

bool head_ok(const HeadArgs &h)
{
    if (!half_type(h.dtype) || h.R < 0 || h.V < 1 || h.D < 1 || h.R > kMost || h.V > kMost || h.D > kMost || h.ldw < h.D || !temperature_ok(h.temperature)) return false;
    if (!h.weight || !aligned(h.weight, 2)) return false;
    if (h.bias && ((h.bias_type != h.dtype && h.bias_type != SPDY_F32) || !aligned(h.bias, type_size(h.bias_type)))) return false;
    if (h.tokens && ((h.index_bits != 32 && h.index_bits != 64) || !aligned(h.tokens, h.index_bits / 8))) return false;
    return h.R == 0 || (h.hidden && aligned(h.hidden, 2) && h.ldh >= h.D);
}

// Whether two matrices of 16-bit elements share memory (rows of one buffer that lie side by side do not, and are not told apart here
// unless their strides are the same).
bool overlap(const void *p, int64_t ldp, int64_t rows_p, const void *q, int64_t ldq, int64_t rows_q, int64_t columns)
{
    if (!p || !q || rows_p <= 0 || rows_q <= 0) return false;
    const uint64_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    const uint64_t a1 = a + static_cast<uint64_t>((rows_p - 1) * ldp + columns) * 2, b1 = b + static_cast<uint64_t>((rows_q - 1) * ldq + columns) * 2;
    if (a1 <= b || b1 <= a) return false;
    if (ldp != ldq) return true;
    const uint64_t stride = static_cast<uint64_t>(ldp) * 2, between = (a > b ? a - b : b - a) % stride;
    return between < static_cast<uint64_t>(columns) * 2 || between > stride - static_cast<uint64_t>(columns) * 2;
}

bool grads_ok(const HeadArgs &h)
{
    if (h.dhidden && h.R > 0 && (!aligned(h.dhidden, 2) || h.lddh < h.D)) return false;
    if (h.dweight && (!aligned(h.dweight, 2) || h.lddw < h.D)) return false;
    return !overlap(h.dhidden, h.lddh, h.R, h.hidden, h.ldh, h.R, h.D) && !overlap(h.dhidden, h.lddh, h.R, h.weight, h.ldw, h.V, h.D) &&
           !overlap(h.dweight, h.lddw, h.V, h.hidden, h.ldh, h.R, h.D) && !overlap(h.dweight, h.lddw, h.V, h.weight, h.ldw, h.V, h.D) &&
           !overlap(h.dweight, h.lddw, h.V, h.dhidden, h.lddh, h.R, h.D);
}

int run(const HeadArgs &h, void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (h.R == 0) {  // gradients of no rows are 0
        if (h.grads && h.dweight) SPDY_EVAL_TRY(cudaMemset2DAsync(h.dweight, static_cast<size_t>(h.lddw) * 2, 0, static_cast<size_t>(h.D) * 2, static_cast<size_t>(h.V), s));
        if (h.grads && h.dbias) SPDY_EVAL_TRY(cudaMemsetAsync(h.dbias, 0, static_cast<size_t>(h.V) * 4, s));
        return SPDY_OK;
    }
    if (!workspace || !aligned(workspace, 256)) return SPDY_ERR_INVALID_ARG;
    if (workspace_bytes < lay_out(h.hidden, h.ldh, h.weight, h.ldw, h.R, h.V, h.D, h.stats, h.grads, h.dbias != nullptr).total) return SPDY_ERR_WORKSPACE_TOO_SMALL;
    return h.dtype == SPDY_BF16 ? run_head<__nv_bfloat16>(h, workspace, s) : run_head<__half>(h, workspace, s);
}

HeadArgs head(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype, const void *bias, int bias_dtype, const void *tokens, int index_bits, int64_t R,
              int64_t V, int64_t D, float temperature)
{
    HeadArgs h = {};
    h.hidden = hidden, h.ldh = ldh, h.weight = weight, h.ldw = ldw, h.dtype = dtype, h.bias = bias, h.bias_type = bias_dtype, h.tokens = tokens, h.index_bits = index_bits;
    h.R = R, h.V = V, h.D = D, h.temperature = temperature;
    return h;
}

}  // namespace

extern "C" {

size_t spdy_linear_token_logprobs_workspace_bytes(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype, int64_t R, int64_t V, int64_t D, int forward,
                                                  int gradients)
{
    if (!half_type(dtype) || R <= 0 || V <= 0 || D <= 0 || R > kMost || V > kMost || D > kMost) return 0;
    return lay_out(hidden, ldh, weight, ldw, R, V, D, forward != 0, gradients != 0, gradients == 2).total;
}

int spdy_linear_token_logprobs(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype, const void *bias, int bias_dtype, const void *tokens, int index_bits,
                               int64_t R, int64_t V, int64_t D, float temperature, float *logprob, float *entropy, float *lse, void *workspace, size_t workspace_bytes,
                               void *cuda_stream)
{
    HeadArgs h = head(hidden, ldh, weight, ldw, dtype, bias, bias_dtype, tokens, index_bits, R, V, D, temperature);
    h.logprob = logprob, h.entropy = entropy, h.lse = lse, h.stats = true;
    if (!head_ok(h) || (R > 0 && logprob && !tokens)) return SPDY_ERR_INVALID_ARG;
    return run(h, workspace, workspace_bytes, cuda_stream);
}

int spdy_linear_token_logprobs_backward(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype, const void *bias, int bias_dtype, const void *tokens,
                                        int index_bits, int64_t R, int64_t V, int64_t D, float temperature, const float *lse, const float *entropy,
                                        const float *grad_logprob, const float *grad_entropy, void *dhidden, int64_t lddh, void *dweight, int64_t lddw, float *dbias,
                                        void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    HeadArgs h = head(hidden, ldh, weight, ldw, dtype, bias, bias_dtype, tokens, index_bits, R, V, D, temperature);
    h.in_lse = lse, h.in_entropy = entropy, h.grad_logprob = grad_logprob, h.grad_entropy = grad_entropy;
    h.dhidden = dhidden, h.lddh = lddh, h.dweight = dweight, h.lddw = lddw, h.dbias = dbias, h.grads = true;
    if (!head_ok(h) || !grads_ok(h)) return SPDY_ERR_INVALID_ARG;
    if (R > 0 && (!lse || (grad_logprob && !tokens) || (grad_entropy && !entropy))) return SPDY_ERR_INVALID_ARG;
    return run(h, workspace, workspace_bytes, cuda_stream);
}

int spdy_linear_token_logprobs_with_grad(const void *hidden, int64_t ldh, const void *weight, int64_t ldw, int dtype, const void *bias, int bias_dtype, const void *tokens,
                                         int index_bits, int64_t R, int64_t V, int64_t D, float temperature, const float *grad_logprob, const float *grad_entropy,
                                         float *logprob, float *entropy, float *lse, void *dhidden, int64_t lddh, void *dweight, int64_t lddw, float *dbias, void *workspace,
                                         size_t workspace_bytes, void *cuda_stream)
{
    HeadArgs h = head(hidden, ldh, weight, ldw, dtype, bias, bias_dtype, tokens, index_bits, R, V, D, temperature);
    h.grad_logprob = grad_logprob, h.grad_entropy = grad_entropy, h.logprob = logprob, h.entropy = entropy, h.lse = lse;
    h.dhidden = dhidden, h.lddh = lddh, h.dweight = dweight, h.lddw = lddw, h.dbias = dbias, h.stats = h.grads = true;
    if (!head_ok(h) || !grads_ok(h) || (R > 0 && (logprob || grad_logprob) && !tokens)) return SPDY_ERR_INVALID_ARG;
    return run(h, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
