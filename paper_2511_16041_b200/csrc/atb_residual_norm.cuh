// Residual norm: what its forward and backward kernels share.  Not part of the ABI.
#pragma once
#include <cuda_runtime.h>

#include "atb_internal.h"
#include "dependent_launch.cuh"
#include "norm_rows.cuh"

namespace residual_norm {

using namespace norm_rows;

struct Weights {
    const void *w, *b, *gate, *pw, *pb;    // each [N] of one type, or NULL
    int w32;                               // that type is FP32, else bf16 (the kernels' TW)
};
struct FwdParams {
    int64_t M, N, ldx, ldf, ldh, ldz;
    const void *x, *f;
    Weights v;
    float scale, eps;
    int center;                            // layer norm, else rms norm
    void *h, *z;
    float* stats;                          // [4][M] (post) or [2][M]: mean and 1 / spread of h, of f; or NULL
};
struct BwdParams {
    int64_t M, N, lddz, lddh, ldx, ldf, lddx, lddf;
    const void *dz, *dh, *x, *f;           // dh may be NULL
    Weights v;
    float scale;
    int center;
    const float* stats;
    void *dx, *df;                         // each may be NULL
    float* part;                           // [walkers][sums][N], or NULL
    int blocks;                            // that walk the rows
};

// Elements n .. n + VEC - 1 of a vector of weights, or `none` where there is no vector.  They are read again for every row, from the L1:
// five of them would take more registers than a row does.
template <class TW, int VEC>
__device__ __forceinline__ void weights(const void* p, int n, float none, float (&v)[VEC]) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = none;
    if (p) {
        Raw<TW, VEC> raw;
        const TW* const at = static_cast<const TW*>(p) + n;
        if constexpr (VEC > 1) {
#pragma unroll
            for (int i = 0; i < static_cast<int>(sizeof(raw.w) / 16); ++i) {
                const uint4 u = __ldg(reinterpret_cast<const uint4*>(at) + i);
                raw.w[4 * i] = u.x; raw.w[4 * i + 1] = u.y; raw.w[4 * i + 2] = u.z; raw.w[4 * i + 3] = u.w;
            }
        } else if constexpr (sizeof(TW) == 4) {
            raw.w[0] = __ldg(reinterpret_cast<const uint32_t*>(at));
        } else {
            raw.w[0] = __ldg(reinterpret_cast<const uint16_t*>(at));
        }
        to_float(raw, v);
    }
}

// A kernel whose rows on their way may take more, with its static arrays, than the 48 KB of shared memory that need no leave.
template <class... Args>
cudaError_t launch_ring(void (*kernel)(Args...), unsigned grid, unsigned block, size_t smem, cudaStream_t stream, Args... args) {
    if (smem > 40 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return e;
    }
    return atb::launch_dependent(kernel, grid, block, 1u, smem, stream, args...);
}

// Types of the stream (x, h and their gradients) and of the branch (f, z and theirs).
enum Types { kBf16 = 0, kMixed = 1, kF32 = 2 };
// Backward: threads of a row and elements of a thread (kWidthCount: the wide kernel), and blocks that stay on an SM.
constexpr int kBlockThreads = 512;         // per SM, 128 registers each
struct Width {
    int threads, elems;
};
constexpr Width kWidths[] = {{32, 8}, {32, 16}, {128, 8}, {256, 8}, {512, 8}, {512, 16}};
constexpr int kWidthCount = 6;
inline int width_of(int64_t N) {
    for (int i = 0; i < kWidthCount; ++i)
        if (N <= static_cast<int64_t>(kWidths[i].threads) * kWidths[i].elems) return i;
    return kWidthCount;
}
__host__ __device__ constexpr int blocks_of(int tpr) { return kBlockThreads / (tpr == 32 ? 128 : tpr); }
// A translation unit for each type of the weights.
cudaError_t launch_forward_f32(const FwdParams& p, Types types, bool vec, bool post, cudaStream_t stream);
cudaError_t launch_forward_bf16(const FwdParams& p, Types types, bool vec, bool post, cudaStream_t stream);
cudaError_t launch_backward_f32(const BwdParams& p, Types types, bool vec, bool post, cudaStream_t stream);
cudaError_t launch_backward_bf16(const BwdParams& p, Types types, bool vec, bool post, cudaStream_t stream);

}  // namespace residual_norm
