// Linear layers (int8 x int8 -> int32, with bias, activation, residual and
// requantization in the epilogue) for gfx950: the folded bias and multipliers,
// and the launches.
#include "linear_plan.h"
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
    for (int k = 16 * lane; k < p.K; k += 16 * 64) {
        const linear::vi4 v = linear::load_tail(row, p.K, k);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = __builtin_amdgcn_sdot4(v[i], 0x01010101, sum, false);
    }
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

hipError_t launch_linear(const LinearArgs& a, hipStream_t stream) {
    using namespace linear;
    switch (plan(a)) {
        case kRows16: launch_rows<1>(a, stream); break;
        case kRows32: launch_rows<2>(a, stream); break;
        case kTile64: launch_tiles<Tile64>(a, stream); break;
        case kTile128: launch_tiles<Tile128>(a, stream); break;
        case kTileW2: launch_tiles<TileW<2>>(a, stream); break;
        case kTileW3: launch_tiles<TileW<3>>(a, stream); break;
        case kTileW4: launch_tiles<TileW<4>>(a, stream); break;
        case kTileW5: launch_tiles<TileW<5>>(a, stream); break;
        case kTile64R: launch_tiles<Tile64R>(a, stream); break;
        case kTile128R: launch_tiles<Tile128R>(a, stream); break;
        case kTile256R: launch_tiles<Tile256R>(a, stream); break;
    }
    return hipGetLastError();
}

}  // namespace fqvit
