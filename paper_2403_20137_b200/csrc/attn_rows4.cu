// The 4-bit instantiations of attn_rows.
#include "attn_rows.cuh"

namespace kvbfp {
kvbfp_status launch_attn_rows4(const AttnArgs& a, int grid, cudaStream_t s) { return launch_attn_p<4>(a, grid, s); }
}  // namespace kvbfp
