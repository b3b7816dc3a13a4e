// Layer norm, forward (values or BFP16 planes) and backward (sm_100a).
//
//   mu = sum(x) / N,  v = sum((x - mu)^2) / N,  r = 1 / sqrt(v + eps),  z = (x - mu) r,  y = z w + b
//   g = dy w,  dx = r (g - sum(g) / N - z sum(g z) / N),  dw = sum over rows of dy z,  db = sum over rows of dy
//
// Bound by memory: the forward pass reads x and writes y, the backward pass reads dy and x and writes dx, and
// nothing else of that size moves.  A row stays in the registers of the threads that share it (TPR threads, up to
// kFwdElems or kBwdElems elements each), so that mean, variance and result take one read; the variance is summed around
// the mean, in a second pass over the registers, since sum(x^2) - N mu^2 loses its digits where |mu| >> sqrt(v).
// All sums are FP32.  Rows wider than the widest kernel are read again for every sum (*_wide kernels).
// Backward: a block walks rows blockIdx.x, + gridDim.x, ...; a thread keeps the same columns for all of them
// and adds dw and db up in registers.  Blocks write their sums to the workspace, a second kernel adds those up in a
// fixed order: no atomics, the same bits on every call.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "atb_internal.h"
#include "bfp16_block.cuh"

namespace {

constexpr int kFwdElems = 32, kBwdElems = 16;     // elements of a row per thread
constexpr int kMaxBlocks = 296;                   // backward: blocks that walk the rows (2 per SM)

// ---------------------------------------------------------------------------------- loads and stores
// VEC consecutive elements as they are in memory, VEC = 8 (16-byte accesses) or 1.
template <class T, int VEC>
struct Raw {
    uint32_t w[VEC * sizeof(T) / 4];
};
template <>
struct Raw<__nv_bfloat16, 1> {
    uint16_t w[1];
};

template <class T, int VEC>
__device__ __forceinline__ void load_raw(const T* p, Raw<T, VEC>& r) {
    if constexpr (VEC == 8) {
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i) {
            const uint4 u = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) + 16 * i);
            r.w[4 * i] = u.x; r.w[4 * i + 1] = u.y; r.w[4 * i + 2] = u.z; r.w[4 * i + 3] = u.w;
        }
    } else if constexpr (sizeof(T) == 4) {
        r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        r.w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
}
template <class T, int VEC>
__device__ __forceinline__ void to_float(const Raw<T, VEC>& r, float (&v)[VEC]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = __uint_as_float(r.w[i]);
    } else if constexpr (VEC == 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
        }
    } else {
        v[0] = __uint_as_float(static_cast<uint32_t>(r.w[0]) << 16);
    }
}
template <class T, int VEC>
__device__ __forceinline__ void load_f(const T* p, float (&v)[VEC]) {
    Raw<T, VEC> r;
    load_raw(p, r);
    to_float(r, v);
}
template <class T, int VEC>
__device__ __forceinline__ void store_f(T* p, const float (&v)[VEC]) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (VEC == 8) {
            reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *p = v[0];
        }
    } else if constexpr (VEC == 8) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b2 = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            o[i] = *reinterpret_cast<const uint32_t*>(&b2);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
    } else {
        *p = __float2bfloat16_rn(v[0]);
    }
}

// ---------------------------------------------------------------------------------- sums over a row's threads
// Every thread of the row gets the sum of K values over the TPR threads.  TPR = 32: one warp; else the whole block,
// through `red`, of which each call of a row takes another slice (a slice is written again only after a
// barrier that follows its last read).
template <int TPR, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float (*red)[K]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) red[warp][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = lane < W ? red[lane][k] : 0.f;
#pragma unroll
            for (int o = W / 2; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
            v[k] = __shfl_sync(0xFFFFFFFFu, v[k], 0);
        }
    }
}

// ---------------------------------------------------------------------------------- forward
struct FwdParams {
    int64_t M, N, ldx, ldy, rows;          // rows: rows the grid covers (M, or M padded for the BFP16 planes)
    const void *x, *w, *b;
    float eps;
    void* y;                               // values, or the mantissa plane
    uint8_t* exp;                          // BFP16: exponent plane
    float *mean, *rstd;
};

// Writes VEC results of row m from column n on: values, or one BFP16 block.
template <class TX, int VEC, bool BFP>
__device__ __forceinline__ void put(const FwdParams& p, int64_t m, int64_t n, const float (&v)[VEC]) {
    if constexpr (BFP) {
        uint32_t packed[2];
        const int E = bfp16::quantize_block8(v, packed);
        *reinterpret_cast<uint2*>(static_cast<int8_t*>(p.y) + m * p.N + n) = make_uint2(packed[0], packed[1]);
        p.exp[((n >> 6) * p.rows + m) * 8 + ((n >> 3) & 7)] = static_cast<uint8_t>(E);
    } else {
        store_f<TX, VEC>(static_cast<TX*>(p.y) + m * p.ldy + n, v);
    }
}
// The exponent plane's padding of row m: blocks past the last column, and whole rows past M.
__device__ __forceinline__ void put_exp_padding(const FwdParams& p, int64_t m, int t, int threads) {
    const int64_t first = m < p.M ? p.N >> 3 : 0, last = ((p.N + 63) >> 6) * 8;
    for (int64_t j = first + t; j < last; j += threads) p.exp[((j >> 3) * p.rows + m) * 8 + (j & 7)] = 0;
}
template <class TX, class TW, int VEC, bool BFP>
__device__ __forceinline__ void scale_and_put(const FwdParams& p, int64_t m, int64_t n, float (&v)[VEC], float mu, float r) {
    float w[VEC], b[VEC];
    if (p.w) load_f<TW, VEC>(static_cast<const TW*>(p.w) + n, w);
    if (p.b) load_f<TW, VEC>(static_cast<const TW*>(p.b) + n, b);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
        v[e] = (v[e] - mu) * r;
        if (p.w) v[e] *= w[e];
        if (p.b) v[e] += b[e];
    }
    put<TX, VEC, BFP>(p, m, n, v);
}

template <class TX, class TW, int VEC, int TPR, bool BFP>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR) layer_norm_kernel(const FwdParams p) {
    constexpr int NV = kFwdElems / VEC, ROWS = TPR == 32 ? 4 : 1;
    __shared__ float red[2][32][1];
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
    const int64_t m = static_cast<int64_t>(blockIdx.x) * ROWS + (TPR == 32 ? threadIdx.x >> 5 : 0);
    if (m >= p.rows) return;                                   // a whole warp (TPR = 32) or a whole block
    if constexpr (BFP) {
        put_exp_padding(p, m, t, TPR);
        if (m >= p.M) return;
    }
    const TX* x = static_cast<const TX*>(p.x) + m * p.ldx;
    Raw<TX, VEC> raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t n = (static_cast<int64_t>(i) * TPR + t) * VEC;
        if (n < p.N) load_raw<TX, VEC>(x + n, raw[i]);
    }
    float s[1] = {0.f}, v[VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((static_cast<int64_t>(i) * TPR + t) * VEC < p.N) {
            to_float(raw[i], v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[0] += v[e];
        }
    const float inv_n = 1.f / static_cast<float>(p.N);
    row_sum<TPR, 1>(s, red[0]);
    const float mu = s[0] * inv_n;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((static_cast<int64_t>(i) * TPR + t) * VEC < p.N) {
            to_float(raw[i], v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[0] += (v[e] - mu) * (v[e] - mu);
        }
    row_sum<TPR, 1>(s, red[1]);
    const float r = rsqrtf(s[0] * inv_n + p.eps);
    if (t == 0) {
        if (p.mean) p.mean[m] = mu;
        if (p.rstd) p.rstd[m] = r;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t n = (static_cast<int64_t>(i) * TPR + t) * VEC;
        if (n < p.N) {
            to_float(raw[i], v);
            scale_and_put<TX, TW, VEC, BFP>(p, m, n, v, mu, r);
        }
    }
}

// Any width: the row is read once for each of mean, variance and result.
template <class TX, class TW, int VEC, bool BFP>
__global__ void __launch_bounds__(1024) layer_norm_wide_kernel(const FwdParams p) {
    __shared__ float red[2][32][1];
    const int64_t m = blockIdx.x;
    if constexpr (BFP) {
        put_exp_padding(p, m, threadIdx.x, 1024);
        if (m >= p.M) return;
    }
    const TX* x = static_cast<const TX*>(p.x) + m * p.ldx;
    float s[1] = {0.f}, v[VEC];
    for (int64_t n = threadIdx.x * VEC; n < p.N; n += 1024 * VEC) {
        load_f<TX, VEC>(x + n, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[0] += v[e];
    }
    const float inv_n = 1.f / static_cast<float>(p.N);
    row_sum<1024, 1>(s, red[0]);
    const float mu = s[0] * inv_n;
    s[0] = 0.f;
    for (int64_t n = threadIdx.x * VEC; n < p.N; n += 1024 * VEC) {
        load_f<TX, VEC>(x + n, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[0] += (v[e] - mu) * (v[e] - mu);
    }
    row_sum<1024, 1>(s, red[1]);
    const float r = rsqrtf(s[0] * inv_n + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[m] = mu;
        if (p.rstd) p.rstd[m] = r;
    }
    for (int64_t n = threadIdx.x * VEC; n < p.N; n += 1024 * VEC) {
        load_f<TX, VEC>(x + n, v);
        scale_and_put<TX, TW, VEC, BFP>(p, m, n, v, mu, r);
    }
}

// ---------------------------------------------------------------------------------- backward
struct BwdParams {
    int64_t M, N, lddy, ldx, lddx;
    const void *dy, *x, *w;
    const float *mean, *rstd;
    void* dx;
    float* part;                           // [blocks][2][N]: sums of dw and db of each block
};

template <class TX, class TW, int VEC, int TPR>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR) layer_norm_backward_kernel(const BwdParams p) {
    constexpr int NV = kBwdElems / VEC, WALKERS = TPR == 32 ? 4 : 1;      // rows a block has in hand at a time
    __shared__ float red[2][32][2];
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
    const int64_t walker = static_cast<int64_t>(blockIdx.x) * WALKERS + (TPR == 32 ? threadIdx.x >> 5 : 0);
    const float inv_n = 1.f / static_cast<float>(p.N);
    float dw[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[i][e] = db[i][e] = 0.f;
    int turn = 0;
    for (int64_t m = walker; m < p.M; m += static_cast<int64_t>(gridDim.x) * WALKERS, turn ^= 1) {
        const TX* x = static_cast<const TX*>(p.x) + m * p.ldx;
        const TX* dy = static_cast<const TX*>(p.dy) + m * p.lddy;
        Raw<TX, VEC> rx[NV], rd[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t n = (static_cast<int64_t>(i) * TPR + t) * VEC;
            if (n < p.N) { load_raw<TX, VEC>(x + n, rx[i]); load_raw<TX, VEC>(dy + n, rd[i]); }
        }
        const float mu = p.mean[m], r = p.rstd[m];
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t n = (static_cast<int64_t>(i) * TPR + t) * VEC;
            if (n < p.N) {
                float vx[VEC], vd[VEC], w[VEC];
                to_float(rx[i], vx);
                to_float(rd[i], vd);
                if (p.w) load_f<TW, VEC>(static_cast<const TW*>(p.w) + n, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float z = (vx[e] - mu) * r, g = p.w ? vd[e] * w[e] : vd[e];
                    s[0] += g;
                    s[1] += g * z;
                    dw[i][e] += vd[e] * z;
                    db[i][e] += vd[e];
                }
            }
        }
        row_sum<TPR, 2>(s, red[turn]);
        const float c0 = s[0] * inv_n, c1 = s[1] * inv_n;
        if (p.dx) {
            TX* dx = static_cast<TX*>(p.dx) + m * p.lddx;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t n = (static_cast<int64_t>(i) * TPR + t) * VEC;
                if (n < p.N) {
                    float vx[VEC], vd[VEC], w[VEC];
                    to_float(rx[i], vx);
                    to_float(rd[i], vd);
                    if (p.w) load_f<TW, VEC>(static_cast<const TW*>(p.w) + n, w);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float z = (vx[e] - mu) * r, g = p.w ? vd[e] * w[e] : vd[e];
                        vx[e] = r * (g - c0 - z * c1);
                    }
                    store_f<TX, VEC>(dx + n, vx);
                }
            }
        }
    }
    if (p.part) {                          // a walker's sums: [walker][2][N]
        float* out = p.part + walker * 2 * p.N;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t n = (static_cast<int64_t>(i) * TPR + t) * VEC;
            if (n < p.N)
#pragma unroll
                for (int e = 0; e < VEC; ++e) { out[n + e] = dw[i][e]; out[p.N + n + e] = db[i][e]; }
        }
    }
}

// Any width, dx: a block per row, which is read for the sums and again for the result.
template <class TX, class TW>
__global__ void __launch_bounds__(1024) layer_norm_backward_wide_kernel(const BwdParams p) {
    __shared__ float red[32][2];
    const int64_t m = blockIdx.x;
    const TX* x = static_cast<const TX*>(p.x) + m * p.ldx;
    const TX* dy = static_cast<const TX*>(p.dy) + m * p.lddy;
    TX* dx = static_cast<TX*>(p.dx) + m * p.lddx;
    const float mu = p.mean[m], r = p.rstd[m], inv_n = 1.f / static_cast<float>(p.N);
    float s[2] = {0.f, 0.f}, vx[1], vd[1], w[1] = {1.f};
    for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
        load_f<TX, 1>(x + n, vx);
        load_f<TX, 1>(dy + n, vd);
        if (p.w) load_f<TW, 1>(static_cast<const TW*>(p.w) + n, w);
        s[0] += vd[0] * w[0];
        s[1] += vd[0] * w[0] * ((vx[0] - mu) * r);
    }
    row_sum<1024, 2>(s, red);
    for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
        load_f<TX, 1>(x + n, vx);
        load_f<TX, 1>(dy + n, vd);
        if (p.w) load_f<TW, 1>(static_cast<const TW*>(p.w) + n, w);
        vx[0] = r * (vd[0] * w[0] - s[0] * inv_n - (vx[0] - mu) * r * (s[1] * inv_n));
        store_f<TX, 1>(dx + n, vx);
    }
}
// Any width, dw and db: a block takes 256 columns and every gridDim.y-th row.
template <class TX>
__global__ void __launch_bounds__(256) layer_norm_backward_columns_kernel(const BwdParams p) {
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (n >= p.N) return;
    float dw = 0.f, db = 0.f, vx[1], vd[1];
    for (int64_t m = blockIdx.y; m < p.M; m += gridDim.y) {
        load_f<TX, 1>(static_cast<const TX*>(p.x) + m * p.ldx + n, vx);
        load_f<TX, 1>(static_cast<const TX*>(p.dy) + m * p.lddy + n, vd);
        dw += vd[0] * ((vx[0] - p.mean[m]) * p.rstd[m]);
        db += vd[0];
    }
    float* out = p.part + static_cast<int64_t>(blockIdx.y) * 2 * p.N;
    out[n] = dw;
    out[p.N + n] = db;
}

// dw[n], db[n] = sum over the `parts` partial sums, in a fixed order: 32 columns of [dw | db] per block, 8 warps that
// take every 8th partial sum, then the 8 in turn.
template <class TW>
__global__ void __launch_bounds__(256) layer_norm_backward_sum_kernel(const float* part, int parts, int64_t N, TW* dw, TW* db) {
    __shared__ float s[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    float v = 0.f;
    if (c < 2 * N)
        for (int i = warp; i < parts; i += 8) v += part[static_cast<int64_t>(i) * 2 * N + c];
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < 2 * N) {
        for (int i = 1; i < 8; ++i) v += s[i][lane];
        TW* out = c < N ? dw : db;
        const float r[1] = {v};
        if (out) store_f<TW, 1>(out + (c < N ? c : c - N), r);
    }
}

// ---------------------------------------------------------------------------------- host
// Threads per row: the fewest of 32, 128, 256, 512, 1024 (forward) that hold a row of N elements; 0: a wide kernel.
int threads_per_row(int64_t N, int elems, int most) {
    for (int t : {32, 128, 256, 512, 1024})
        if (t <= most && N <= static_cast<int64_t>(t) * elems) return t;
    return 0;
}

template <class TX, class TW, int VEC, bool BFP>
void launch_fwd(const FwdParams& p, cudaStream_t st) {
    const unsigned rows = static_cast<unsigned>(p.rows), quads = static_cast<unsigned>((p.rows + 3) / 4);
    switch (threads_per_row(p.N, kFwdElems, 1024)) {
        case 32: layer_norm_kernel<TX, TW, VEC, 32, BFP><<<quads, 128, 0, st>>>(p); break;
        case 128: layer_norm_kernel<TX, TW, VEC, 128, BFP><<<rows, 128, 0, st>>>(p); break;
        case 256: layer_norm_kernel<TX, TW, VEC, 256, BFP><<<rows, 256, 0, st>>>(p); break;
        case 512: layer_norm_kernel<TX, TW, VEC, 512, BFP><<<rows, 512, 0, st>>>(p); break;
        case 1024: layer_norm_kernel<TX, TW, VEC, 1024, BFP><<<rows, 1024, 0, st>>>(p); break;
        default: layer_norm_wide_kernel<TX, TW, VEC, BFP><<<rows, 1024, 0, st>>>(p);
    }
}

// Blocks that walk the rows: enough to fill the SMs, and at least 4 rows for each walker, whose sums of 8 N bytes
// go through the workspace.
int walking_blocks(int64_t M, int64_t N) {
    const int tpr = threads_per_row(N, kBwdElems, 512);
    const int64_t walkers = tpr == 32 ? 4 : 1;
    int64_t blocks = (M + 4 * walkers - 1) / (4 * walkers);
    if (blocks > kMaxBlocks) blocks = kMaxBlocks;
    return static_cast<int>(blocks < 1 ? 1 : blocks);
}
int partial_sums(int64_t M, int64_t N) {
    return walking_blocks(M, N) * (threads_per_row(N, kBwdElems, 512) == 32 ? 4 : 1);
}

template <class TX, class TW, int VEC>
void launch_bwd(const BwdParams& p, cudaStream_t st) {
    const unsigned blocks = static_cast<unsigned>(walking_blocks(p.M, p.N));
    switch (threads_per_row(p.N, kBwdElems, 512)) {
        case 32: layer_norm_backward_kernel<TX, TW, VEC, 32><<<blocks, 128, 0, st>>>(p); break;
        case 128: layer_norm_backward_kernel<TX, TW, VEC, 128><<<blocks, 128, 0, st>>>(p); break;
        case 256: layer_norm_backward_kernel<TX, TW, VEC, 256><<<blocks, 256, 0, st>>>(p); break;
        case 512: layer_norm_backward_kernel<TX, TW, VEC, 512><<<blocks, 512, 0, st>>>(p); break;
        default:
            if (p.dx) layer_norm_backward_wide_kernel<TX, TW><<<static_cast<unsigned>(p.M), 1024, 0, st>>>(p);
            if (p.part)
                layer_norm_backward_columns_kernel<TX><<<dim3(static_cast<unsigned>((p.N + 255) / 256), blocks), 256, 0, st>>>(p);
    }
}

bool known_type(int t) { return t == ATB_F32 || t == ATB_BF16; }
int64_t size_of(int t) { return t == ATB_F32 ? 4 : 2; }
bool aligned_to(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }
bool vec_ok(const void* p, int64_t ld, int type) { return atb::aligned16(p) && ld * size_of(type) % 16 == 0; }

atb_status_t check_common(int64_t M, int64_t N, int x_type, int w_type) {
    if (!known_type(x_type) || !known_type(w_type))
        return atb::fail(ATB_ERR_BAD_ARGUMENT, "x_type=%d, w_type=%d: ATB_F32 or ATB_BF16", x_type, w_type);
    if (M < 0 || N < 0 || M > 0x7FFFFFFFll - 32 || N > (1ll << 30))
        return atb::fail(ATB_ERR_BAD_SHAPE, "need 0 <= M < 2^31 - 32 and 0 <= N <= 2^30 (got %lld, %lld)", (long long)M, (long long)N);
    return ATB_OK;
}

#define ATB_LN_TYPES(CALL)                                                                     \
    if (x_type == ATB_F32 && w_type == ATB_F32) { CALL(float, float); }                        \
    else if (x_type == ATB_F32) { CALL(float, __nv_bfloat16); }                                \
    else if (w_type == ATB_F32) { CALL(__nv_bfloat16, float); }                                \
    else { CALL(__nv_bfloat16, __nv_bfloat16); }

atb_status_t forward(int64_t M, int64_t N, int x_type, const void* X, int64_t ldx, int w_type, const void* W, const void* B,
                     float eps, void* Y, int64_t ldy, uint8_t* exp, float* mean, float* rstd, void* stream) {
    atb::clear_error();
    atb_status_t s = check_common(M, N, x_type, w_type);
    if (s != ATB_OK) return s;
    if (!(eps >= 0.f)) return atb::fail(ATB_ERR_BAD_ARGUMENT, "eps must be >= 0");
    if (exp && N % 8 != 0) return atb::fail(ATB_ERR_BAD_SHAPE, "N=%lld is not a multiple of the block size 8", (long long)N);
    if (M == 0 || N == 0) return ATB_OK;
    if (!X || !Y) return atb::fail(ATB_ERR_NULL_POINTER, "the input and the output must be non-NULL");
    if (ldx < N || (!exp && ldy < N)) return atb::fail(ATB_ERR_BAD_SHAPE, "ldx=%lld and ldy=%lld must be >= N", (long long)ldx, (long long)ldy);
    if (!aligned_to(X, size_of(x_type)) || !aligned_to(W, size_of(w_type)) || !aligned_to(B, size_of(w_type)) ||
        (!exp && !aligned_to(Y, size_of(x_type))) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements");
    const bool vec = N % 8 == 0 && vec_ok(X, ldx, x_type) && atb::aligned16(W) && atb::aligned16(B) && (exp || vec_ok(Y, ldy, x_type));
    if (exp && (!vec || !atb::aligned16(Y) || !atb::aligned16(exp)))
        return atb::fail(ATB_ERR_MISALIGNED, "BFP16 output needs 16-byte aligned pointers and rows of X");
    int sms = 0;
    s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    FwdParams p{M, N, ldx, ldy, exp ? atb::round_up(M, 32) : M, X, W, B, eps, Y, exp, mean, rstd};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
#define ATB_LN_BFP(TX, TW) launch_fwd<TX, TW, 8, true>(p, st)
#define ATB_LN_VEC(TX, TW) launch_fwd<TX, TW, 8, false>(p, st)
#define ATB_LN_ONE(TX, TW) launch_fwd<TX, TW, 1, false>(p, st)
    if (exp) { ATB_LN_TYPES(ATB_LN_BFP) }
    else if (vec) { ATB_LN_TYPES(ATB_LN_VEC) }
    else { ATB_LN_TYPES(ATB_LN_ONE) }
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "layer norm launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

}  // namespace

extern "C" atb_status_t atb_layer_norm(int64_t M, int64_t N, int x_type, const void* X_dev, int64_t ldx, int w_type,
                                       const void* W_dev, const void* B_dev, float eps, void* Y_dev, int64_t ldy,
                                       float* mean_dev, float* rstd_dev, void* stream) {
    return forward(M, N, x_type, X_dev, ldx, w_type, W_dev, B_dev, eps, Y_dev, ldy, nullptr, mean_dev, rstd_dev, stream);
}

extern "C" atb_status_t atb_layer_norm_bfp16(int64_t M, int64_t N, int x_type, const void* X_dev, int64_t ldx, int w_type,
                                             const void* W_dev, const void* B_dev, float eps, int8_t* mant_dev, uint8_t* exp_dev,
                                             float* mean_dev, float* rstd_dev, void* stream) {
    if (M > 0 && N > 0 && !exp_dev) {
        atb::clear_error();
        return atb::fail(ATB_ERR_NULL_POINTER, "the exponent plane must be non-NULL");
    }
    // an empty call passes a non-NULL plane on, so that it is checked as a BFP16 call
    return forward(M, N, x_type, X_dev, ldx, w_type, W_dev, B_dev, eps, mant_dev, N, exp_dev ? exp_dev : reinterpret_cast<uint8_t*>(16),
                   mean_dev, rstd_dev, stream);
}

extern "C" size_t atb_layer_norm_backward_workspace_bytes(int64_t M, int64_t N) {
    if (M < 0 || N < 1) return 0;
    return static_cast<size_t>(partial_sums(M, N)) * 2 * static_cast<size_t>(N) * sizeof(float);
}

extern "C" atb_status_t atb_layer_norm_backward(int64_t M, int64_t N, int x_type, const void* dY_dev, int64_t lddy, const void* X_dev,
                                                int64_t ldx, int w_type, const void* W_dev, const float* mean_dev, const float* rstd_dev,
                                                void* dX_dev, int64_t lddx, void* dW_dev, void* dB_dev,
                                                void* workspace_dev, size_t workspace_bytes, void* stream) {
    atb::clear_error();
    atb_status_t s = check_common(M, N, x_type, w_type);
    if (s != ATB_OK) return s;
    if (N == 0) return ATB_OK;
    const bool sums = dW_dev || dB_dev;
    if (M > 0 && (!dY_dev || !X_dev || !mean_dev || !rstd_dev))
        return atb::fail(ATB_ERR_NULL_POINTER, "dY, X, mean and rstd must be non-NULL");
    if (sums && !workspace_dev) return atb::fail(ATB_ERR_NULL_POINTER, "dW and dB need the workspace");
    if (M > 0 && (ldx < N || lddy < N || (dX_dev && lddx < N)))
        return atb::fail(ATB_ERR_BAD_SHAPE, "lddy=%lld, ldx=%lld and lddx=%lld must be >= N", (long long)lddy, (long long)ldx, (long long)lddx);
    if (!aligned_to(X_dev, size_of(x_type)) || !aligned_to(dY_dev, size_of(x_type)) || !aligned_to(dX_dev, size_of(x_type)) ||
        !aligned_to(W_dev, size_of(w_type)) || !aligned_to(dW_dev, size_of(w_type)) || !aligned_to(dB_dev, size_of(w_type)) ||
        !aligned_to(mean_dev, 4) || !aligned_to(rstd_dev, 4) || !aligned_to(workspace_dev, 16))
        return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements, the workspace to 16 bytes");
    if (sums && workspace_bytes < atb_layer_norm_backward_workspace_bytes(M, N))
        return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes,
                         atb_layer_norm_backward_workspace_bytes(M, N));
    int sms = 0;
    s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    BwdParams p{M, N, lddy, ldx, lddx, dY_dev, X_dev, W_dev, mean_dev, rstd_dev, dX_dev, sums ? static_cast<float*>(workspace_dev) : nullptr};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = N % 8 == 0 && vec_ok(X_dev, ldx, x_type) && vec_ok(dY_dev, lddy, x_type) && atb::aligned16(W_dev) &&
                     (!dX_dev || vec_ok(dX_dev, lddx, x_type));
    if (M > 0 && (dX_dev || sums)) {
#define ATB_LN_BWD_VEC(TX, TW) launch_bwd<TX, TW, 8>(p, st)
#define ATB_LN_BWD_ONE(TX, TW) launch_bwd<TX, TW, 1>(p, st)
        if (vec) { ATB_LN_TYPES(ATB_LN_BWD_VEC) }
        else { ATB_LN_TYPES(ATB_LN_BWD_ONE) }
    }
    if (sums) {
        const unsigned blocks = static_cast<unsigned>((2 * N + 31) / 32);
        const int parts = M > 0 ? partial_sums(M, N) : 0;
        if (w_type == ATB_F32)
            layer_norm_backward_sum_kernel<float><<<blocks, 256, 0, st>>>(p.part, parts, N, static_cast<float*>(dW_dev), static_cast<float*>(dB_dev));
        else
            layer_norm_backward_sum_kernel<__nv_bfloat16><<<blocks, 256, 0, st>>>(p.part, parts, N, static_cast<__nv_bfloat16*>(dW_dev),
                                                                                  static_cast<__nv_bfloat16*>(dB_dev));
    }
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "layer norm backward launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}
