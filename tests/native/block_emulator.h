// Runs a block's device code on the CPU, each thread a fiber, so that orders in which a GPU seldom runs its warps can be had on
// purpose: a warp runs until all of its threads stand at a block barrier (or are done), then the next one of a given order; its
// lanes one after another, from the last one where the order begins with the last warp.
// Warp-wide operations meet the warp's threads.  Barriers of a block that do not pair (threads of one block standing at different
// ones, or some gone while others wait) are reported.
#ifndef BLOCK_EMULATOR_H
#define BLOCK_EMULATOR_H

#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include <ucontext.h>

#include <functional>
#include <string>
#include <vector>

namespace emulator {

struct Index {
    unsigned x;
};

struct Fiber {
    ucontext_t context;
    std::vector<char> stack;
    int barrier = 0;        // the line of the block barrier it stands at, 0 for none
    bool in_warp = false;   // stands in a warp-wide operation
    bool done = false;
    uint64_t given = 0;     // what it brings to that operation
};

struct Block {
    std::vector<Fiber> fibers;
    ucontext_t scheduler;
    std::function<void()> body;
    unsigned current = 0;
};

inline Block *&block()
{
    static Block *b = nullptr;
    return b;
}
inline Index here() { return {block()->current}; }
inline Fiber &fiber() { return block()->fibers[block()->current]; }
inline void yield() { swapcontext(&fiber().context, &block()->scheduler); }

inline void block_barrier(int line)
{
    fiber().barrier = line;
    yield();
}

// All 32 values of the warp, once all of its threads are here.
inline std::vector<uint64_t> meet(uint64_t mine)
{
    fiber().given = mine;
    fiber().in_warp = true;
    yield();
    const unsigned first = block()->current / 32 * 32;
    std::vector<uint64_t> all(32);
    for (unsigned l = 0; l < 32; ++l) all[l] = block()->fibers[first + l].given;
    fiber().in_warp = true;  // nobody brings the next value before all have read these
    yield();
    return all;
}

inline void entry()
{
    block()->body();
    fiber().done = true;
    for (;;) yield();
}

// Runs `body` as a block of `threads`, warps in the order of `order` between barriers; an empty text, or what went wrong.
inline std::string run(int threads, const std::vector<int> &order, std::function<void()> body)
{
    Block b;
    block() = &b;
    b.body = body;
    b.fibers.resize(threads);
    for (Fiber &f : b.fibers) {
        f.stack.resize(64 << 10);
        getcontext(&f.context);
        f.context.uc_stack.ss_sp = f.stack.data();
        f.context.uc_stack.ss_size = f.stack.size();
        f.context.uc_link = nullptr;
        makecontext(&f.context, entry, 0);
    }
    for (;;) {
        for (int w : order) {
            for (;;) {
                bool ran = false;
                for (int i = 0; i < 32; ++i) {
                    const int l = order[0] * 32 + 32 == threads ? 31 - i : i;
                    Fiber &f = b.fibers[w * 32 + l];
                    if (f.done || f.barrier || f.in_warp) continue;
                    b.current = w * 32 + l;
                    swapcontext(&b.scheduler, &f.context);
                    ran = true;
                }
                if (ran) continue;
                int meeting = 0;
                for (int l = 0; l < 32; ++l) meeting += b.fibers[w * 32 + l].in_warp;
                if (meeting == 0) break;
                if (meeting != 32) return "threads of a warp are missing from a warp-wide operation";
                for (int l = 0; l < 32; ++l) b.fibers[w * 32 + l].in_warp = false;
            }
        }
        int done = 0, line = 0;
        for (const Fiber &f : b.fibers) {
            if (f.done) {
                ++done;
                continue;
            }
            if (line && line != f.barrier) return "threads stand at different barriers: lines " + std::to_string(line) + " and " + std::to_string(f.barrier);
            line = f.barrier;
        }
        if (done == threads) return "";
        if (done) return "some threads are gone while others stand at the barrier of line " + std::to_string(line);
        for (Fiber &f : b.fibers) f.barrier = 0;
    }
}

}  // namespace emulator

// ---------------------------------------------------------------------------------------------- the language of device code
#define __device__
#define __forceinline__ inline
#define __noinline__ __attribute__((noinline))
#define threadIdx emulator::here()
#define __syncthreads() emulator::block_barrier(__LINE__)

struct uint4 {
    uint32_t x, y, z, w;
};
inline uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return {x, y, z, w}; }
inline float __uint_as_float(uint32_t b)
{
    float f;
    memcpy(&f, &b, 4);
    return f;
}
inline uint32_t __float_as_uint(float f)
{
    uint32_t b;
    memcpy(&b, &f, 4);
    return b;
}
inline int __popc(uint32_t b) { return __builtin_popcount(b); }
inline uint32_t atomicAdd(uint32_t *p, uint32_t v)
{
    const uint32_t old = *p;
    *p += v;
    return old;
}
inline uint32_t __reduce_max_sync(uint32_t, uint32_t v)
{
    for (uint64_t o : emulator::meet(v)) v = o > v ? static_cast<uint32_t>(o) : v;
    return v;
}
inline uint32_t __reduce_min_sync(uint32_t, uint32_t v)
{
    for (uint64_t o : emulator::meet(v)) v = o < v ? static_cast<uint32_t>(o) : v;
    return v;
}
inline int __reduce_add_sync(uint32_t, int v)
{
    int sum = 0;
    for (uint64_t o : emulator::meet(static_cast<uint32_t>(v))) sum += static_cast<int>(o);
    return sum;
}
inline int __shfl_up_sync(uint32_t, int v, int d)
{
    const unsigned lane = threadIdx.x % 32;
    const std::vector<uint64_t> all = emulator::meet(static_cast<uint32_t>(v));
    return lane >= static_cast<unsigned>(d) ? static_cast<int>(all[lane - d]) : v;
}
template <class T> inline T min(T a, T b) { return b < a ? b : a; }
template <class T> inline T max(T a, T b) { return a < b ? b : a; }

#endif
