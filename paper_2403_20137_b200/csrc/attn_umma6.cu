// The 6-bit instantiations of umma_prep and attn_umma.
#include "attn_umma.cuh"

namespace kvbfp {
kvbfp_status launch_attn_umma6(const AttnArgs& a, int grid, cudaStream_t s) { return launch_umma_p<6>(a, grid, s); }
}  // namespace kvbfp
