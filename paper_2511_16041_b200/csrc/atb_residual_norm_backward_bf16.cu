// Residual norm, backward, with bf16 vectors of weights.
#include "residual_norm_backward.cuh"

namespace residual_norm {

cudaError_t launch_backward_bf16(const BwdParams& p, Types types, bool vec, bool post, cudaStream_t stream) { return launch_backward<__nv_bfloat16>(p, types, vec, post, stream); }

}  // namespace residual_norm
