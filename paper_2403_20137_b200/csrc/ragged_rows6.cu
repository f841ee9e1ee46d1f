// The 6-bit instantiations of ragged_rows.
#include "ragged_rows.cuh"

namespace kvbfp {
kvbfp_status launch_ragged_rows6(const RaggedArgs& a, int grid, cudaStream_t s) { return launch_ragged_p<6>(a, grid, s); }
}  // namespace kvbfp
