// Which kernel and tile a product in 8 bits takes: a rule on its sizes, for the launch and for what checks that every tile is tested.
#pragma once

namespace tst {

constexpr int kStepK = 128;   // of K that a workgroup takes at a time

// Which kernel and tile.  With all of them the busiest compute unit loads some 65 GB/s, over all sizes measured (no limit of the hardware: a copy
// of tiles through the LDS moves 110), so the choice is the one for which it loads least: rounds of workgroups x bytes of a workgroup, and for
// k_w8_rows the sums that its wavefronts exchange.  Measured with K = N = 4096 (us): 256 rows 11.8 with 64 x 64 tiles of k_w8_rows, 23 with k_w8_tiles<4>,
// 31 with k_w8_tiles<8>; 512 rows 20 / 24 / 31; 1024 rows 36 / 24 / 32; 2048 rows 70 / 38 / 36; 4096 rows 61 with k_w8_tiles<8>, 72
// with <4>.  64 x 16384 x 4096: 17.3 with 32 x 32 tiles of k_w8_rows, 18.3 with 64 x 16, 26 with 64 x 64.
struct GemmTile {
    bool rows;
    int mt, nt;   // 16 mt rows x 16 nt columns
};
constexpr GemmTile kGemmTiles[] = {{true, 1, 1}, {true, 1, 2}, {true, 2, 2}, {true, 4, 2}, {true, 4, 4}, {false, 4, 16}, {false, 8, 16}};

inline GemmTile choose_tile(int M, int K, int N, int compute_units)
{
    const auto blocks = [](int n, int size) { return n / size + (n % size != 0); };
    const double steps = blocks(K, kStepK);
    GemmTile best = kGemmTiles[0];
    double least = 1e300;
    for (const GemmTile &t : kGemmTiles) {
        const double groups = (double)blocks(M, 16 * t.mt) * blocks(N, 16 * t.nt);
        const double rounds = groups > compute_units ? (double)(long long)((groups + compute_units - 1) / compute_units) : 1;
        const double x_rows = M < 16 * t.mt ? M : 16 * t.mt;
        const double bytes = rounds * (steps * kStepK * (x_rows + 16 * t.nt) + (t.rows ? 20e3 + 6e3 * t.mt * t.nt : 0));
        if (bytes < least) {
            least = bytes;
            best = t;
        }
    }
    return best;
}

}  // namespace tst
