// The 6-bit instantiations of ragged_umma.
#include "ragged_umma.cuh"

namespace kvbfp {
kvbfp_status launch_ragged_umma6(const RaggedArgs& a, int grid, cudaStream_t s) {
    return a.fmt.block == 16 ? launch_prompt<6, true>(a, grid, s) : launch_prompt<6, false>(a, grid, s);
}
}  // namespace kvbfp
