// Which scales and biases the waves of a product's tiles read (compiled and run by test_product_reads_cpu.py; no device code, no
// GPU): every index lies inside the array, whichever wave of whichever tile forms it.
#include <cstdio>
#include "lnmod_launch.hpp"

using namespace lnmod;

struct TileShape {
    int bm, bn, wm, wn;
};
constexpr TileShape kShapes[] = {{32, 32, 2, 1},  {32, 64, 2, 2},   {64, 64, 2, 2},   {96, 64, 2, 2},   {128, 64, 2, 2},
                                 {128, 128, 4, 2}, {128, 128, 2, 2}, {128, 256, 2, 4}, {256, 256, 2, 4}};

int main() {
    long bad = 0, idle = 0, read = 0;
    const int64_t sizes[] = {1, 2, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 95, 97, 127, 128, 129, 161, 255, 257, 300, 385, 600};
    for (const TileShape& t : kShapes) {
        const int rows = t.bm / t.wm, features = t.bn / t.wn;
        for (const int64_t M : sizes) {
            for (const int64_t N : sizes) {
                ProductArgs a{};
                a.M = M;
                a.N = N;
                deal_tiles(a, t.bm, t.bn);
                for (int64_t m0 = 0; m0 < int64_t(a.tiles_m) * t.bm; m0 += rows) {
                    for (int64_t n0 = 0; n0 < int64_t(a.tiles_n) * t.bn; n0 += features) {
                        if (!has_outputs(a, m0, n0)) {
                            ++idle;
                            continue;
                        }
                        const int most_m = last_of(M, m0, rows), most_n = last_of(N, n0, features);
                        for (int i = 0; i < rows; ++i, ++read) {
                            const int64_t m = m0 + held(i, most_m);
                            bad += m < m0 || m >= M || (m0 + i < M && m != m0 + i);
                        }
                        for (int j = 0; j < features; ++j, ++read) {
                            const int64_t n = n0 + held(j, most_n);
                            bad += n < n0 || n >= N || (n0 + j < N && n != n0 + j);
                            if (j % 8 == 0 && j + 7 <= most_n) bad += n0 + j + 7 >= N;        // eight at a time
                        }
                    }
                }
            }
        }
    }
    std::printf("%ld reads, %ld waves without outputs, %ld failures\n", read, idle, bad);
    return bad == 0 && idle > 0 ? 0 : 1;
}
