// Few-row products with an epilogue, 3 plane(s).
#include "linear_rows_launch.hpp"

namespace splitee_host {

int launch_linear_rows_bf16x3(const splitee::LinArgs& p, bool tiled, const LinPlan& plan, hipStream_t s)
{
    return tiled ? rows_bm<3, true>(p, plan, s) : rows_bm<3, false>(p, plan, s);
}

}  // namespace splitee_host
