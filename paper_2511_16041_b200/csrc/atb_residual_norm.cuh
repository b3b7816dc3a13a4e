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

// A thread's elements in eights, as four pairs: a group of VEC = 8, or eight single elements.
template <class T, int VEC>
__device__ __forceinline__ void pairs_of(const Raw<T, VEC> (&r)[8 / VEC], float2 (&v)[4]) {
    if constexpr (VEC == 8) {
        float f[8];
        to_float(r[0], f);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = make_float2(f[2 * k], f[2 * k + 1]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float a[1], b[1];
            to_float(r[2 * k], a);
            to_float(r[2 * k + 1], b);
            v[k] = make_float2(a[0], b[0]);
        }
    }
}
// Where they are: eight c of a thread whose first column is `col`.  Elements past the row's end are 0, as are their weights.
template <int VEC, int TPR>
struct Eight {
    static constexpr int G = 8 / VEC;      // groups
    int N, col, c;
    __device__ __forceinline__ int n(int g) const { return col + (c * G + g) * TPR * VEC; }
    __device__ __forceinline__ bool in(int g) const { return n(g) < N; }
    template <class T, class Source>
    __device__ __forceinline__ void read(const Source& src, int stage, int64_t m, float2 (&v)[4]) const {
        Raw<T, VEC> r[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (in(g)) src.read(stage, m, c * G + g, r[g]);
            else clear(r[g]);
        }
        pairs_of(r, v);
    }
    template <class T>
    __device__ __forceinline__ void load(const void* row, float2 (&v)[4]) const {
        Raw<T, VEC> r[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (in(g)) load_raw<T, VEC>(static_cast<const T*>(row) + n(g), r[g]);
            else clear(r[g]);
        }
        pairs_of(r, v);
    }
    // ... of a vector of weights.
    template <class TW>
    __device__ __forceinline__ void weight(const void* w, float none, float2 (&v)[4]) const {
        float f[G][VEC];
#pragma unroll
        for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[g][e] = 0.f;
            if (in(g)) weights<TW, VEC>(w, n(g), none, f[g]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = VEC == 8 ? make_float2(f[0][(2 * k) % VEC], f[0][(2 * k + 1) % VEC]) : make_float2(f[(2 * k) % G][0], f[(2 * k + 1) % G][0]);
    }
    template <class T>
    __device__ __forceinline__ void store(void* row, const float2 (&v)[4]) const {
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (in(g)) {
                float f[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int k = g * VEC + e;
                    f[e] = k & 1 ? v[k / 2].y : v[k / 2].x;
                }
                store_f<T, VEC>(static_cast<T*>(row) + n(g), f);
            }
    }
};

// A vector of weights at a thread's CH eights.  KEEP: in registers, loaded once, as they are in memory (single elements: in FP32); else read
// again wherever they are used.
template <class TW, int VEC, int TPR, int CH, bool KEEP>
struct Vector {
    const void* p;
    float none;
    Raw<TW, 8> raw[KEEP && VEC == 8 ? CH : 1];
    float2 one[KEEP && VEC == 1 ? CH : 1][4];
    __device__ __forceinline__ Vector(const void* p_, float none_, int N, int col) : p(p_), none(none_) {
        if constexpr (KEEP) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const Eight<VEC, TPR> at{N, col, c};
                if constexpr (VEC == 8) {
                    load_or<TW, 8>(static_cast<const TW*>(p), at.n(0), N, none, raw[c]);
                } else {
                    at.template weight<TW>(p, none, one[c]);
#pragma unroll
                    for (int k = 0; k < 4; ++k)      // kept: not converted again in every row
                        asm volatile("" : "+f"(one[c][k].x), "+f"(one[c][k].y));
                }
            }
        }
    }
    __device__ __forceinline__ void get(const Eight<VEC, TPR>& at, float2 (&v)[4]) const {
        if constexpr (!KEEP) {
            at.template weight<TW>(p, none, v);
        } else if constexpr (VEC == 8) {
            const Raw<TW, 8> r[1] = {raw[at.c]};
            pairs_of<TW, 8>(r, v);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = one[at.c][k];
        }
    }
};

// A kernel whose rows on their way take more than the 48 KB of shared memory that need no leave is given it once per device.
template <auto KERNEL, class Params>
cudaError_t launch_ring(unsigned grid, unsigned block, size_t smem, cudaStream_t stream, const Params& p) {
    const cudaError_t e = atb::allow_shared_memory<KERNEL>(smem);
    return e != cudaSuccess ? e : atb::launch_dependent(KERNEL, grid, block, 1u, smem, stream, p);
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
