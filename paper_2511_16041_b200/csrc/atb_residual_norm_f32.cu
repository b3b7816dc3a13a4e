// Residual norm, forward, with FP32 vectors of weights.
#include "residual_norm_forward.cuh"

namespace residual_norm {

cudaError_t launch_forward_f32(const FwdParams& p, Types types, bool vec, bool post, cudaStream_t stream) { return launch_forward<float>(p, types, vec, post, stream); }

}  // namespace residual_norm
