// The 4-bit instantiations of umma_prep and attn_umma.
#include "attn_umma.cuh"

namespace kvbfp {
kvbfp_status launch_attn_umma4(const AttnArgs& a, int grid, cudaStream_t s) { return launch_umma_p<4>(a, grid, s); }
}  // namespace kvbfp
