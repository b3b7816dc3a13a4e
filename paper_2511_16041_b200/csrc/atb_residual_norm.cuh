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
    int w32;                               // that type is FP32, else bf16
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
};

// Elements n .. n + VEC - 1 of a vector of weights, or `none` where there is no vector.  They are read again for every row, from the L1:
// five of them would take more registers than a row does.
template <int VEC>
__device__ __forceinline__ void weights(const void* p, int w32, int n, float none, float (&v)[VEC]) {
    if (!p) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = none;
    } else if constexpr (VEC == 1) {
        v[0] = w32 ? __ldg(static_cast<const float*>(p) + n) : __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const uint16_t*>(p) + n)) << 16);
    } else if (w32) {
#pragma unroll
        for (int i = 0; i < VEC / 4; ++i) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(p) + n) + i);
            v[4 * i] = f.x; v[4 * i + 1] = f.y; v[4 * i + 2] = f.z; v[4 * i + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC / 8; ++i) {
            const uint4 u = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + n) + i);
            const uint32_t q[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[8 * i + 2 * e] = __uint_as_float(q[e] << 16);
                v[8 * i + 2 * e + 1] = __uint_as_float(q[e] & 0xFFFF0000u);
            }
        }
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
// sums: of the rows' products that the weights' gradients are made of
inline int sums_per_column(bool post) { return post ? 4 : 3; }
int walkers(int64_t M, int64_t N);
cudaError_t launch_backward(const BwdParams& p, Types types, bool vec, bool post, cudaStream_t stream);

}  // namespace residual_norm
