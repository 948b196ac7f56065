// The search for a row's largest elements (csrc/eval_top.cuh) by a block that runs on the CPU, its warps in many orders, against
// a sorted list.  Prints what went wrong; exit status 0 if nothing did.
#include "block_emulator.h"

#include <math.h>

#include <algorithm>
#include <random>

#define SPDY_TOP_MAX 128

namespace spdy_eval {

inline float neg_inf() { return -INFINITY; }
inline float quiet_nan() { return NAN; }

struct Half16 {  // the upper half of a float
    uint16_t bits;
};
template <class T> struct Elem;
template <> struct Elem<float> {
    static constexpr int kVec = 4;
    static float to_float(float x) { return x; }
    static float from_float(float x) { return x; }
    static void unpack(uint4 r, float *f) { memcpy(f, &r, 16); }
};
template <> struct Elem<Half16> {
    static constexpr int kVec = 8;
    static float to_float(Half16 x) { return __uint_as_float(static_cast<uint32_t>(x.bits) << 16); }
    static Half16 from_float(float x) { return {static_cast<uint16_t>(__float_as_uint(x) >> 16)}; }
    static void unpack(uint4 r, float *f)
    {
        uint16_t h[8];
        memcpy(h, &r, 16);
        for (int i = 0; i < 8; ++i) f[i] = to_float({h[i]});
    }
};
template <class T> uint4 load_part(const T *p, int n, int e)
{
    T v[Elem<T>::kVec];
    for (int i = 0; i < Elem<T>::kVec; ++i) v[i] = e + i >= 0 && e + i < n ? p[e + i] : Elem<T>::from_float(neg_inf());
    uint4 r;
    memcpy(&r, v, 16);
    return r;
}
template <class T> uint4 load_stream(const T *p) { return load_part(p, Elem<T>::kVec, 0); }
template <class T> struct Row {
    const T *p;
    int n, lead;
    int granules() const { return (n + lead + Elem<T>::kVec - 1) / Elem<T>::kVec; }
    int first(int g) const { return g * Elem<T>::kVec - lead; }
    uint4 load(int g) const { return load_part(p, n, first(g)); }
};

}  // namespace spdy_eval

#include "../../paper_2201_13096_b200/csrc/eval_top.cuh"

using namespace spdy_eval;

namespace {

constexpr int kGroupSteps = 32, U = 4;
int failures = 0;

template <class T, int NT> void one(const std::vector<float> &values, int lead, int parts, int part, int want, const std::vector<int> &order, const char *what)
{
    std::vector<T> x;
    for (float v : values) x.push_back(Elem<T>::from_float(v));
    const Row<T> row{x.data(), static_cast<int>(x.size()), lead};
    const int per = (row.granules() + parts - 1) / parts, steps = (per - 1) / (NT * U) + 1;
    const int g0 = std::min(row.granules(), part * per), g1 = std::min(row.granules(), g0 + per);
    const int e0 = std::max(0, row.first(g0)), e1 = std::min(row.n, row.first(g1));
    want = std::max(0, std::min(want, e1 - e0));
    if (want == 0) return;
    int shift = 0;
    while (steps >> shift >= kGroupSteps) ++shift;
    const int groups = (steps + (1 << shift) - 1) >> shift;
    std::vector<float> largest(static_cast<size_t>(groups) * NT, NAN);
    for (int s = 0; s < steps; ++s)
        for (int t = 0; t < NT; ++t) {
            float all = NAN;
            for (int u = 0; u < U; ++u) {
                const int g = g0 + s * NT * U + u * NT + t;
                float f[8];
                for (int i = 0; i < 8; ++i) f[i] = neg_inf();
                if (g < g1) Elem<T>::unpack(row.load(g), f);
                for (int i = 0; i < Elem<T>::kVec; ++i) all = fmaxf(all, f[i]);
            }
            if (g0 + s * NT * U + t >= g1) all = NAN;
            float &to = largest[(s >> shift) * NT + t];
            to = s & ((1 << shift) - 1) ? fmaxf(all, to) : all;
        }
    static TopShared sh;
    memset(&sh, 0xa5, sizeof sh);  // shared memory holds anything at first
    const std::string wrong = emulator::run(NT, order, [&] { find_top<T, NT, U>(sh, largest.data(), groups, shift, row, g0, g1, want); });
    std::vector<uint64_t> keys;
    for (int e = e0; e < e1; ++e) keys.push_back(rank_key(Elem<T>::to_float(x[e]), static_cast<uint32_t>(e)));
    std::sort(keys.rbegin(), keys.rend());
    const bool same = std::equal(sh.best, sh.best + want, keys.begin());
    if (wrong.empty() && same) return;
    if (++failures <= 10)
        printf("%s, %zu elements of %zu bytes, lead %d, part %d of %d, best %d, %d threads, first warp %d: %s\n", what, x.size(), sizeof(T), lead, part, parts, want, NT, order[0],
               wrong.empty() ? "other elements than the largest" : wrong.c_str());
}

template <class T, int NT> void orders(const std::vector<float> &values, int lead, int parts, int part, int want, std::mt19937 &rng, const char *what)
{
    std::vector<int> order(NT / 32);
    for (int w = 0; w < NT / 32; ++w) order[w] = w;
    one<T, NT>(values, lead, parts, part, want, order, what);
    std::reverse(order.begin(), order.end());
    one<T, NT>(values, lead, parts, part, want, order, what);
    std::shuffle(order.begin(), order.end(), rng);
    one<T, NT>(values, lead, parts, part, want, order, what);
}

}  // namespace

int main()
{
    std::mt19937 rng(7);
    std::normal_distribution<float> normal;
    const char *kinds[] = {"normal", "constant", "rising", "two values", "mostly masked", "all masked", "NaN among them", "all NaN", "large at the end"};
    const int sizes[] = {1, 5, 700, 2100, 9000, 20011, 70001};
    for (int k = 0; k < 9; ++k)
        for (int n : sizes) {
            std::vector<float> v(n);
            for (int i = 0; i < n; ++i) {
                const float r = normal(rng);
                v[i] = k == 0 ? r : k == 1 ? 1.5f : k == 2 ? 1e-3f * static_cast<float>(i) : k == 3 ? static_cast<float>(i % 3 == 0) : k == 4 ? (rng() % 50 ? neg_inf() : r)
                     : k == 5 ? neg_inf() : k == 6 ? (i % 5 == 3 ? NAN : r) : k == 7 ? NAN : (i > n - n / 50 ? 4.f + r : r);
            }
            for (int want : {1, 20, 128}) {
                const int lead = static_cast<int>(rng() % 8);
                orders<Half16, 128>(v, lead, 1, 0, want, rng, kinds[k]);
                orders<float, 128>(v, lead % 4, 1, 0, want, rng, kinds[k]);
                if (n > 9000) orders<Half16, 128>(v, lead, 4, n % 4, want, rng, kinds[k]);
            }
        }
    if (failures) printf("%d of the runs failed\n", failures);
    return failures != 0;
}
