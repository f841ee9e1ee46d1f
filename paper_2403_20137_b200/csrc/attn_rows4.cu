// The 4-bit instantiations of attn_rows.
#include "attn_rows.cuh"

namespace kvbfp {
kvbfp_status launch_attn_rows4(const AttnArgs& a, cudaStream_t s) { return launch_attn_p<4>(a, s); }
}  // namespace kvbfp
