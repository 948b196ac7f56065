// The order of tiles and the division it rests on (csrc/eval_ranges.h): every tile of every share comes once, in groups; quotients are
// exact up to the ends of 32 bits.
#include <stdio.h>

#include <initializer_list>
#include <vector>

#include "../../paper_2201_13096_b200/csrc/eval_ranges.h"

using spdy_eval::Divisor;
using spdy_eval::Tiles;

int main()
{
    int failures = 0;
    uint64_t state = 88172645463325252ull;
    const auto next = [&] { return state ^= state << 13, state ^= state >> 7, state ^= state << 17; };
    const auto check = [&](uint32_t x, uint32_t d) {
        if (Divisor(d).of(x) != x / d && ++failures <= 10) printf("%u / %u gives %u\n", x, d, Divisor(d).of(x));
    };
    for (uint32_t d = 1; d <= 4000; ++d)
        for (uint32_t x : {0u, 1u, d - 1, d, d + 1, 2 * d - 1, 0xffffffffu, 0xffffffffu / d * d, 0xffffffffu / d * d - 1}) check(x, d);
    for (int k = 0; k < 3000000; ++k) {
        const uint32_t d = static_cast<uint32_t>(next() >> (33 + next() % 31)) | 1u, x = static_cast<uint32_t>(next());
        check(x, d), check(x / d * d, d), check(x / d * d - 1, d), check(x, d + 1);
    }
    for (int m : {1, 2, 3, 7, 8, 9, 16, 31, 33})
        for (int n : {1, 2, 3, 5, 74})
            for (int group : {1, 3, 8, 4096})
                for (int shares : {1, 2, 5}) {
                    const Tiles tiles(m, n, group);
                    std::vector<int> seen(static_cast<size_t>(m) * n * shares, 0);
                    if (tiles.count() != static_cast<uint32_t>(m) * n) ++failures;
                    int before = -1;
                    for (uint32_t item = 0; item < tiles.count() * shares; ++item) {
                        int share, tm, tn;
                        tiles.at(item, share, tm, tn);
                        if (share < 0 || share >= shares || tm < 0 || tm >= m || tn < 0 || tn >= n) {
                            if (++failures <= 10) printf("%d x %d by %d, %d shares: item %u is (%d, %d) of %d\n", m, n, group, shares, item, tm, tn, share);
                            continue;
                        }
                        ++seen[(static_cast<size_t>(share) * m + tm) * n + tn];
                        const int place = share * m + tm / tiles.group * tiles.group;  // shares and groups do not interleave
                        if (place < before) ++failures;
                        before = place;
                    }
                    for (int c : seen)
                        if (c != 1 && ++failures <= 10) printf("%d x %d by %d, %d shares: a tile comes %d times\n", m, n, group, shares, c);
                }
    // the largest grid a launch takes
    const Tiles large(1 << 15, (1 << 15) - 1, 4096);
    int share, tm, tn;
    large.at(large.count() - 1, share, tm, tn);
    if (share != 0 || tm != (1 << 15) - 1 || tn != (1 << 15) - 2) ++failures, printf("the last tile is (%d, %d)\n", tm, tn);
    return failures != 0;
}
