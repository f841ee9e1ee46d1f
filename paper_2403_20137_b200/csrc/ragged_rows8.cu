// The 8-bit instantiations of ragged_rows.
#include "ragged_rows.cuh"

namespace kvbfp {
kvbfp_status launch_ragged_rows8(const RaggedArgs& a, int grid, cudaStream_t s) { return launch_ragged_p<8>(a, grid, s); }
}  // namespace kvbfp
