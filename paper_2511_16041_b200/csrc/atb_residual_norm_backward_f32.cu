// Residual norm, backward, with FP32 vectors of weights.
#include "residual_norm_backward.cuh"

namespace residual_norm {

cudaError_t launch_backward_f32(const BwdParams& p, Types types, bool vec, bool post, cudaStream_t stream) { return launch_backward<float>(p, types, vec, post, stream); }

}  // namespace residual_norm
