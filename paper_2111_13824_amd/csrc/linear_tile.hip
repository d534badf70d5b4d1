// Instances of the linear layers' tile kernel: one shape of the tile a
// translation unit.
#include "linear_tile.h"

namespace fqvit {
namespace linear {
namespace {

template <class S, int ACT, bool RES, bool ACC>
void go(const LinearArgs& a, hipStream_t stream) {
    const int tiles_n = (a.N + S::BN - 1) / S::BN;
    const unsigned tiles = (unsigned)((a.T + S::BT - 1) / S::BT * tiles_n);
    launch_kernel(linear_tile_kernel<S, ACT, RES, ACC>, dim3(tiles), dim3(S::threads), 0, stream, a,
                  tiles_n, tiles);
}

}  // namespace

template <class S>
void launch_tiles(const LinearArgs& a, hipStream_t stream) {
    const bool res = a.residual != nullptr;
    if (a.acc)
        go<S, FQ_ACT_NONE, false, true>(a, stream);
    else if (a.act == FQ_ACT_TABLE)
        res ? go<S, FQ_ACT_TABLE, true, false>(a, stream) : go<S, FQ_ACT_TABLE, false, false>(a, stream);
    else if (a.act == FQ_ACT_RELU)
        res ? go<S, FQ_ACT_RELU, true, false>(a, stream) : go<S, FQ_ACT_RELU, false, false>(a, stream);
    else
        res ? go<S, FQ_ACT_NONE, true, false>(a, stream) : go<S, FQ_ACT_NONE, false, false>(a, stream);
}

#if defined(FQ_TILE_W)
template void launch_tiles<TileW<FQ_TILE_W>>(const LinearArgs&, hipStream_t);
#elif defined(FQ_TILE_256R)
template void launch_tiles<Tile256R>(const LinearArgs&, hipStream_t);
#elif defined(FQ_TILE_128)
template void launch_tiles<Tile128>(const LinearArgs&, hipStream_t);
template void launch_tiles<Tile128R>(const LinearArgs&, hipStream_t);
#else
template void launch_tiles<Tile64>(const LinearArgs&, hipStream_t);
template void launch_tiles<Tile64R>(const LinearArgs&, hipStream_t);
#endif

}  // namespace linear
}  // namespace fqvit
