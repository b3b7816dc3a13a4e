// Residual norm, forward, with bf16 vectors of weights.
#include "residual_norm_forward.cuh"

namespace residual_norm {

cudaError_t launch_forward_bf16(const FwdParams& p, Types types, bool vec, bool post, cudaStream_t stream) { return launch_forward<__nv_bfloat16>(p, types, vec, post, stream); }

}  // namespace residual_norm
