// The 4-bit instantiations of ragged_rows.
#include "ragged_rows.cuh"

namespace kvbfp {
kvbfp_status launch_ragged_rows4(const RaggedArgs& a, int grid, cudaStream_t s) { return launch_ragged_p<4>(a, grid, s); }
}  // namespace kvbfp
