// Tiles of products with an epilogue, 1 plane(s).
#include "linear_tile_launch.hpp"

namespace splitee_host {

int launch_linear_tile_bf16(const splitee::LinArgs& p, bool tiled, const LinPlan& plan, float* part, hipStream_t s)
{
    return tiled ? tile_size<1, true>(p, plan, part, s) : tile_size<1, false>(p, plan, part, s);
}

}  // namespace splitee_host
