// Which kernel a linear layer's product takes (host code only).
#pragma once

#include "layers_internal.h"

namespace fqvit {
namespace linear {

enum Kernel {
    kRows16,        // linear_rows.hip: 16 rows of x a workgroup, 32
    kRows32,
    kTile64,        // linear_tile.h: channels x rows 64 x 64, 128 x 128,
    kTile128,
    kTileW2,        // 256 x 128, 256 x 192, 256 x 256, 256 x 320
    kTileW3,
    kTileW4,
    kTileW5,
    kTile64R,       // 64 x 64, 128 x 128, 256 x 256 with the loads through registers
    kTile128R,
    kTile256R,
};

// Few rows: the kernels that share the inputs out among the wavefronts of a workgroup
// (16 channels x 16 or 32 rows) finish a product sooner than tiles of 64 x 64, which take
// K one step after another, until their workgroups come to several a CU.  Microseconds,
// fitted to 160 products (T 33 .. 1576, K 192 .. 8192, N 64 .. 4096): 0.2% over the
// fastest of the three, where tiles alone took 26% more.  K = 4096, N = 1024: 5.9 in 16
// rows, 7.7 in 32 and 10.2 in tiles for T = 48, 9.5, 7.8 and 10.7 for 96, 15.5, 13.2 and
// 10.9 for 197; K = 768, N = 192: 3.1, 3.4 and 4.2 for 197, 4.4, 4.4 and 4.3 for 788.
// Without whole units: K = 1001, N = 300: 4.5, 5.6 and 7.9 for 197, 9.8, 8.4 and 8.0 for 788.
struct FewCost {
    float fixed, round, input;      // round + input K: 256 workgroups more
};
constexpr FewCost kFew[2][3] = {    // 16 rows, 32 rows, a round of tiles of 64 x 64
    {{2.3f, 0.08f, 1.9e-3f}, {2.25f, 0.14f, 2.8e-3f}, {2.9f, 0.0f, 4.8e-3f}},
    {{2.3f, 0.08f, 0.85e-3f}, {2.25f, 0.14f, 1.22e-3f}, {2.9f, 0.0f, 1.8e-3f}},     // whole units
};

// What a tile costs, fitted to measurements of 136 products (T 64 .. 25088, K 192 ..
// 32768, N 192 .. 10240, operands that were not read just before): `per` workgroups
// share a CU; a CU's tiles take per round of `per` fixed + input K microseconds, the
// share `few` of it at least.  Large tiles move fewer bytes through L2 for a product
// but fill the last round worse:
// 9232 x 1024 x 4096 takes 45 us in 464 tiles of 256 x 320 and 53 in 592 of 256 x 256
// (48 with a table, which the fit leaves out, as it does residuals); 9232 x 4096 x 1024
// takes 40 us in 196 tiles of 256 x 192 and 44 in 148 of 256 x 256 (42 with a residual);
// 12608 x 768 x 2304 takes 30 us in 450 tiles of 256 x 256 and 34 in 360 of 256 x 320;
// 788 x 768 x 768 takes 4.3 us in 156 tiles of 64 x 64 and 13 in 12 of 256 x 256.
// Over the 136 the choice costs 0.05% more than the fastest tile of each.
struct Cost {
    int bn, bt, per;
    float few, fixed, input;
};
constexpr Cost kCosts[] = {
    {64, 64, 3, 0.33f, 2.5f, 4.6e-3f},    {128, 128, 2, 0.73f, 2.4f, 7.4e-3f},
    {256, 128, 2, 0.64f, 3.2f, 12.4e-3f}, {256, 192, 1, 1.0f, 3.1f, 8.0e-3f},
    {256, 256, 1, 1.0f, 3.7f, 10.2e-3f},  {256, 320, 1, 1.0f, 4.3f, 10.2e-3f},
};

// The same for the loads through registers (99 products, K 47 .. 4091, N 101 .. 4097):
// 9232 x 1021 x 4097 takes 81 us in tiles of 256 x 256, 100 in 128 x 128 and 143 in 64
// x 64; 788 x 1021 x 1021 9.3 in 64 x 64, 15 in 128 x 128 and 25 in 256 x 256.
constexpr Cost kCostsR[] = {
    {64, 64, 3, 0.51f, 2.1f, 14.1e-3f},
    {128, 128, 2, 0.92f, 7.6f, 9.1e-3f},
    {256, 256, 1, 1.0f, 7.3f, 13.0e-3f},
};

template <int shapes>
int cheapest(const LinearArgs& a, const Cost (&costs)[shapes]) {
    int best = 0;
    float least = 0;
    for (int i = 0; i < shapes; ++i) {
        const Cost& c = costs[i];
        const int64_t tiles = ((a.N + c.bn - 1) / c.bn) * ((a.T + c.bt - 1) / c.bt);
        const float share = (float)((tiles + 255) / 256) / (float)c.per;
        const float cost = (share > c.few ? share : c.few) * (c.fixed + c.input * (float)a.K);
        if (i == 0 || cost < least) {
            best = i;
            least = cost;
        }
    }
    return best;
}

inline int64_t ceil_div(int64_t a, int b) { return (a + b - 1) / b; }

// Up to 32 rows the tiles are one line of them, and their time is the weights' way to
// the chip: fixed + K (input + tile times the number of tiles of 64 x 64), in
// microseconds, fitted to products of weights that come from HBM (K 192 .. 4096, N 1024
// .. 65536).  The kernels of few rows reach memory sooner, but their rounds cost more
// than their weights once there are several: K = 1024, 16 and 32 rows: 3.6 and 4.0 us for
// N = 4096 (tiles 4.9), 5.6 and 7.2 for 12288 (6.3), 11.4 and 16.5 for 32768 (9.4).
// Up to 8 rows they keep up with the tiles for most N (2 rows of K = 1024, N = 65536: 15.9
// us, tiles 18.3).  Fitted to 402 products of 1 to 32 rows (1.1% over the fastest kernel of
// each, 24% at most); on 103 others (K to 20000, N to 120000) 2.4% over it, where the
// kernels of few rows alone took 15% more, and 2.4 times as long at most.
struct LineCost {
    float fixed, input, tile;
};
constexpr LineCost kLine[2] = {{3.6f, 6.6e-3f, 1.95e-5f}, {4.1f, 2.06e-3f, 1.66e-6f}};   // whole units

// Rows of whole 16-byte units on 16-byte aligned bases can be loaded straight into
// LDS.
inline Kernel plan(const LinearArgs& a) {
    const bool units = a.K % 16 == 0 &&
                       ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15) == 0;
    if (a.T <= 8) return kRows16;
    const int64_t tiles = ceil_div(a.T, 64) * ceil_div(a.N, 64);
    if (a.T <= 32 || tiles <= 256) {
        float cost[3];
        for (int i = 0; i < 3; ++i) {
            const FewCost& c = kFew[units][i];
            const int64_t blocks = i < 2 ? ceil_div(a.N, 16) * ceil_div(a.T, 16 << i) : 1;
            cost[i] = c.fixed + (float)ceil_div(blocks, 256) * (c.round + c.input * (float)a.K);
        }
        const LineCost& l = kLine[units];
        if (a.T <= 32) cost[2] = l.fixed + (float)a.K * (l.input + l.tile * (float)tiles);
        if (cost[0] < cost[2] || cost[1] < cost[2]) return cost[0] < cost[1] ? kRows16 : kRows32;
        // most rows of a larger tile would be empty (16 rows of K = 464, N = 93454: 16.2 us,
        // 19.4 in 128 x 128; 17 of K = 1001, N = 65537: 27.1 and 33.5)
        if (a.T <= 32) return units ? kTile64 : kTile64R;
    }
    return units ? (Kernel)(kTile64 + cheapest(a, kCosts))
                 : (Kernel)(kTile64R + cheapest(a, kCostsR));
}

}  // namespace linear
}  // namespace fqvit
