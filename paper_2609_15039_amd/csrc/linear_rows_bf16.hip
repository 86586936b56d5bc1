// Few-row products with an epilogue, 1 plane(s).
#include "linear_rows_launch.hpp"

namespace splitee_host {

int launch_linear_rows_bf16(const splitee::LinArgs& p, bool tiled, const LinPlan& plan, hipStream_t s)
{
    return tiled ? rows_bm<1, true>(p, plan, s) : rows_bm<1, false>(p, plan, s);
}

}  // namespace splitee_host
