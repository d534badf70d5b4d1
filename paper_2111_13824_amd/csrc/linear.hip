// Linear layers (int8 x int8 -> int32, with bias, activation, residual and
// requantization in the epilogue) for gfx950: the folded bias and multipliers,
// and which kernel a product takes.
#include "linear_tile.h"

namespace fqvit {
namespace {

using linear::kBlock;

// ---------------------------------------------------------------------------
// Folded bias and multipliers: a wavefront a channel
// ---------------------------------------------------------------------------

__global__ __launch_bounds__(kBlock) void linear_fold_kernel(LinearFoldArgs p) {
    const int n = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6);
    if (n >= p.N) return;
    const int lane = threadIdx.x & 63;
    const int8_t* row = p.w + (int64_t)n * p.K;
    int sum = 0;
    for (int k = lane; k < p.K; k += 64) sum += row[k];
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane != 0) return;
    const double s_w = (double)p.s_w[n];
    const bool live = s_w > 0.0 && isfinite(s_w);
    const double s_n = (double)p.s_x * s_w;
    double b = live && p.bias ? (double)p.bias[n] / s_n : 0.0;
    b = b == b ? fmin(fmax(rint(b), -1073741824.0), 1073741824.0) : 0.0;
    p.fold[n] = (int)b - p.zp_x * sum;
    if (p.mul) p.mul[n] = live ? (float)fmin(s_n / (double)p.s_y, 3.4028234663852886e38) : 0.0f;
}

}  // namespace

hipError_t launch_linear_fold(const LinearFoldArgs& a, hipStream_t stream) {
    launch_kernel(linear_fold_kernel, dim3((unsigned)((a.N + 3) / 4)), dim3(kBlock), 0, stream, a);
    return hipGetLastError();
}

namespace {

// What a tile costs, from measurements of 90 products (T 64 .. 25088, K 192 .. 4096,
// N 192 .. 4096): `per` workgroups a CU, a round of tiles on all CUs takes
// fixed + input K microseconds, and a round that is not full the share `few` of
// it at least.  Large tiles move fewer bytes through L2 for a product but fill the
// last round worse: 9232 x 1024 x 4096 takes 47 us in 464 tiles of 256 x 320, 55 in
// 592 of 256 x 256 and 55 in 2336 of 128 x 128; 9232 x 4096 x 1024 takes 42 us in 196
// tiles of 256 x 192, 48 in 148 of 256 x 256; 12608 x 768 x 2304 takes 31 us in 450
// tiles of 256 x 256, 35 in 360 of 256 x 320; 1576 x 768 x 768 takes 4.8 us in 300
// tiles of 64 x 64, 12.9 in 21 of 256 x 256.  Over the 90 the choice costs 0.2% more
// than the fastest tile of each.
struct Cost {
    int bn, bt, per;
    float few, fixed, input;
};
constexpr Cost kCosts[] = {
    {64, 64, 3, 0.33f, 1.1f, 4.6e-3f},  {128, 128, 2, 0.82f, 1.9f, 6.9e-3f},
    {256, 128, 1, 1.0f, 2.0f, 7.1e-3f}, {256, 192, 1, 1.0f, 2.7f, 9.0e-3f},
    {256, 256, 1, 1.0f, 4.0f, 11.1e-3f}, {256, 320, 1, 1.0f, 6.5f, 12.5e-3f},
};

// Products of so few rows take the kernel that shares the inputs out among the
// wavefronts of a workgroup: K = 4096, N = 1024: 4.5 us for one row (9.0 in tiles of
// 64 x 64), 7.3 for 32 (9.2), 8.5 for 33 (9.3), 9.8 for 48 (9.2).
constexpr int kFewRows = 32;

int choose(const LinearArgs& a, int shapes) {
    int best = 0;
    float least = 0;
    for (int i = 0; i < shapes; ++i) {
        const Cost& c = kCosts[i];
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

}  // namespace

hipError_t launch_linear(const LinearArgs& a, hipStream_t stream) {
    using namespace linear;
    if (a.T <= kFewRows) {
        launch_rows(a, stream);
    } else if (a.K % 16 == 0 &&
        ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15) == 0) {
        switch (choose(a, 6)) {
            case 0: launch_tiles<Tile64>(a, stream); break;
            case 1: launch_tiles<Tile128>(a, stream); break;
            case 2: launch_tiles<TileW<2>>(a, stream); break;
            case 3: launch_tiles<TileW<3>>(a, stream); break;
            case 4: launch_tiles<TileW<4>>(a, stream); break;
            default: launch_tiles<TileW<5>>(a, stream); break;
        }
    } else {
        choose(a, 2) == 0 ? launch_tiles<Tile64R>(a, stream) : launch_tiles<Tile128R>(a, stream);
    }
    return hipGetLastError();
}

}  // namespace fqvit
