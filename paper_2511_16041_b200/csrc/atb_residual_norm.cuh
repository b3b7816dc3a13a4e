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

// Elements n .. n + VEC - 1 of a vector of weights, or `none` where there is no vector.  (Where they are kept between rows: Vector, below.)
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
// The first FULL groups of a thread lie inside every row that the kernel gets.
template <int VEC, int TPR, int FULL>
struct Eight {
    static constexpr int G = 8 / VEC;      // groups
    int N, col, c;
    __device__ __forceinline__ int n(int g) const { return col + (c * G + g) * TPR * VEC; }
    __device__ __forceinline__ bool in(int g) const { return c * G + g < FULL || n(g) < N; }
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

// A vector of weights at a thread's CH eights, or the product of two.  Elements past the row's end are 0.
//   kRead: read again wherever it is used;  kKept: in registers, loaded once, as it is in memory (single elements and products: in FP32);
//   kShared: in shared memory in FP32, each thread's own 16-byte pieces at `place`
enum Place { kRead = 0, kKept = 1, kShared = 2 };
template <class TW, int VEC, int TPR, int CH, int FULL, int PLACE, bool PRODUCT = false>
struct Vector {
    static constexpr bool RAW = PLACE == kKept && VEC == 8 && !PRODUCT, VALUES = PLACE == kKept && !RAW;
    static constexpr uint32_t PIECES = (TPR == 32 ? 128 : TPR) * 16, BYTES = CH * 2 * PIECES;
    const void *p, *q;
    float none, none_q;
    uint32_t place;
    Raw<TW, 8> raw[RAW ? CH : 1];
    float2 value[VALUES ? CH : 1][4];
    using At = Eight<VEC, TPR, FULL>;
    __device__ __forceinline__ Vector(int N, int col, const void* p_, float none_, const void* q_ = nullptr, float none_q_ = 1.f, uint32_t place_ = 0)
        : p(p_), q(q_), none(none_), none_q(none_q_), place(place_ + threadIdx.x * 16) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const At at{N, col, c};
            if constexpr (RAW) {
                load_or<TW, 8>(static_cast<const TW*>(p), at.n(0), N, none, raw[c]);
            } else if constexpr (VALUES) {
                read(at, value[c]);
#pragma unroll
                for (int k = 0; k < 4; ++k)          // kept: not made again in every row
                    asm volatile("" : "+f"(value[c][k].x), "+f"(value[c][k].y));
            } else if constexpr (PLACE == kShared) {
                float2 v[4];
                read(at, v);
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(place + (c * 2 + half) * PIECES), "f"(v[2 * half].x), "f"(v[2 * half].y),
                                 "f"(v[2 * half + 1].x), "f"(v[2 * half + 1].y) : "memory");
            }
        }
    }
    __device__ __forceinline__ void read(const At& at, float2 (&v)[4]) const {
        at.template weight<TW>(p, none, v);
        if constexpr (PRODUCT) {
            float2 f[4];
            at.template weight<TW>(q, none_q, f);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], f[k]);
        }
    }
    __device__ __forceinline__ void get(const At& at, float2 (&v)[4]) const {
        if constexpr (RAW) {
            const Raw<TW, 8> r[1] = {raw[at.c]};
            pairs_of<TW, 8>(r, v);
        } else if constexpr (VALUES) {
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = value[at.c][k];
        } else if constexpr (PLACE == kShared) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[2 * half].x), "=f"(v[2 * half].y), "=f"(v[2 * half + 1].x), "=f"(v[2 * half + 1].y)
                             : "r"(place + (at.c * 2 + half) * PIECES));
        } else {
            read(at, v);
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
// Backward: threads of a row and elements of a thread (kWidthCount: the wide kernel), and blocks that stay on an SM.  Eight elements while 512
// threads last: beside sixteen, four sums a column leave the weights no registers (30000 x 512 bf16 with a norm of f, 32 threads of
// sixteen 178 us, 64 of eight 72 us; without it 68 and 57 us).
constexpr int kBlockThreads = 512;         // per SM, 128 registers each
struct Width {
    int threads, elems;
};
constexpr int kWidthCount = 10;
constexpr Width kWidths[kWidthCount] = {{32, 8}, {64, 8}, {96, 8}, {128, 8}, {192, 8}, {256, 8}, {384, 8}, {512, 8}, {384, 16}, {512, 16}};
// Groups of a thread that lie inside every row of a width: the rows are wider than the width before it takes.
__host__ __device__ constexpr int full_of(int threads, int elems, int vec, int fewer) {
    const int groups = vec > 1 ? 0 : fewer / threads;
    return groups < elems ? groups : elems;
}
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
