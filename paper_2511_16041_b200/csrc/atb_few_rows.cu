// Products of one or two rows (M <= kFewRows) with a weight matrix stored [K][N] (sm_100a):
//   y = x W, or with two matrices of one shape  h = act(x Wg) * (x Wu).
//
// Bound by memory: every weight is read once, for 2 M operations.  A cluster of CTAs takes COLS = 64 or 32 columns (128 or 64
// bytes of a weight row, or of a row of each of the two); its CTAs' warps deal the K rows out among themselves: a thread
// holds 8 columns and 8 consecutive rows at a time, so that 8 (16) loads of 16 bytes are in flight per thread before the
// first is used, and its 8 values of each row of x come in one load.  The sums of a thread (FP32) are joined over the
// row groups of the warp by shuffles, over the warps in shared memory and over the cluster through distributed shared
// memory, always in the same order: no second kernel, no workspace, no atomics.
// Measured: one row through a block of 4096 x 10944 (269 MB of weights) 46 us, 5.8 TB/s, 0.89 of the measured copy rate; the
// second product's first weights are fetched while the first product drains.  The tensor-core products, with 128 rows of
// which one is real, take 57 us for it; which form takes how many rows, and both measured: kFewRows.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>

#include "atb_few_rows.h"
#include "dependent_launch.cuh"
#include "glu.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int kWarps = 4, kThreads = kWarps * 32;

struct FewParams {
    int64_t K, N, ldx, ldw, ldy;
    const __nv_bfloat16 *x, *w0, *w1;
    __nv_bfloat16* y;
    void *g, *u;                           // the two products themselves, FP32 with keep32, else bf16, or NULL
    int64_t ldg;
    int M, act, keep32;
    int weights_settled;                   // the weights are not written by the kernel before this one on the stream
    // the linear layer's epilogue: y = act(z) + r, z = x W + bias; y and r FP32 with y32
    const void *bias, *r;
    int64_t ldr;
    void *out, *z;                         // z [M][N]
    int y32, bias32, z32;
};

// CTAs per SM (launch bounds): what leaves every thread the registers for its loads in flight (32 per matrix) and its sums
// (8 per row and matrix).  Measured at 4096 x 10944, one row, block of both products: 6 for NW = 1: 46.4 us, 7: 50.4 us, 5: 46.9 us;
// NW = 2 with 5 instead of 4: 51.2 us, with 3: 53.9 us.  One fewer of each (5 and 3; 4 for two rows) at other sizes, one row and two:
// 512 x 1024 6.3 and 6.8 us instead of 6.3 and 7.0, 2048 x 5464 18.6 and 20.2 instead of 17.5 and 19.0, 8192 x 24576 188 and 202
// instead of 194 and 208; one more spills, and takes 239 us for one row of the last (212 as it is, both on a cold L2).
constexpr int resident(int MT, int NW) { return NW == 2 ? 4 : MT == 1 ? 6 : 5; }


__device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint4 load_stream(const __nv_bfloat16* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

__device__ __forceinline__ float value_at(const void* p, int64_t at, int fp32) {
    return fp32 ? static_cast<const float*>(p)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at]);
}
__device__ __forceinline__ void value_to(void* p, int64_t at, int fp32, float v) {
    if (fp32) static_cast<float*>(p)[at] = v;
    else static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
}
// What the linear layer makes of the product v of row m and column n.
__device__ __forceinline__ void finish_linear(const FewParams& p, int m, int64_t n, float v) {
    if (p.bias) v += value_at(p.bias, n, p.bias32);
    if (p.z) value_to(p.z, m * p.N + n, p.z32, v);
    glu::with_linear_act(p.act, [&](auto act) { v = glu::act_value<act.value>(make_float2(v, v)).x; });
    if (p.r) v += value_at(p.r, m * p.ldr + n, p.y32);
    value_to(p.out, m * p.ldy + n, p.y32, v);
}

// LINEAR (NW = 1): finish_linear instead of a bf16 store.
template <int MT, int NW, int COLS, bool LINEAR>
__global__ void __launch_bounds__(kThreads, resident(MT, NW)) few_rows_kernel(const FewParams p) {
    constexpr int LANES = COLS / 8, SUBS = 32 / LANES, ROUND = kWarps * SUBS * 8;      // rows that a CTA takes at a time
    __shared__ __align__(16) float sums[kWarps][MT * NW][COLS];
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LANES;
    const int64_t col0 = static_cast<int64_t>(blockIdx.x / ranks) * COLS, col = col0 + (lane % LANES) * 8;

    float acc[NW][MT][8];
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[w][m][e] = 0.f;

    uint4 w[NW][8];
    int64_t k = static_cast<int64_t>(rank) * ROUND + (warp * SUBS + sub) * 8;
    const auto load = [&] {                // K is a multiple of 8: all 8 rows exist
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[0][i] = load_stream(p.w0 + (k + i) * p.ldw + col);
            if constexpr (NW == 2) w[1][i] = load_stream(p.w1 + (k + i) * p.ldw + col);
        }
    };
    const bool mine = col < p.N;           // N is a multiple of 8
    // Weights that were complete before the kernel ahead of this one started may be fetched while it still runs.
    if (p.weights_settled) {
        if (mine && k < p.K) load();
        sm100::grid_dependency_wait();
    } else {
        sm100::grid_dependency_wait();
        if (mine && k < p.K) load();
    }
    sm100::grid_dependency_launch();
    uint4 xv[MT];
    const auto load_x = [&] {
#pragma unroll
        for (int m = 0; m < MT; ++m)
            xv[m] = *reinterpret_cast<const uint4*>(p.x + m * p.ldx + k);
    };
    if (mine) {
        if (k < p.K) load_x();
        while (k < p.K) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int n = 0; n < NW; ++n) {
                    const uint32_t ww[4] = {w[n][i].x, w[n][i].y, w[n][i].z, w[n][i].w};
                    float f[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) { f[2 * e] = lo(ww[e]); f[2 * e + 1] = hi(ww[e]); }
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const uint32_t xw = i < 2 ? xv[m].x : i < 4 ? xv[m].y : i < 6 ? xv[m].z : xv[m].w;
                        const float xf = i & 1 ? hi(xw) : lo(xw);
#pragma unroll
                        for (int e = 0; e < 8; ++e) acc[n][m][e] = fmaf(xf, f[e], acc[n][m][e]);
                    }
                }
            }
            k += static_cast<int64_t>(ranks) * ROUND;
            if (k < p.K) { load(); load_x(); }
        }
    }
    // the row groups of the warp
#pragma unroll
    for (int n = 0; n < NW; ++n)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int o = LANES; o < 32; o <<= 1) acc[n][m][e] += __shfl_xor_sync(0xFFFFFFFFu, acc[n][m][e], o);
            }
            if (sub == 0) {
                float4* dst = reinterpret_cast<float4*>(&sums[warp][n * MT + m][lane * 8]);
                dst[0] = make_float4(acc[n][m][0], acc[n][m][1], acc[n][m][2], acc[n][m][3]);
                dst[1] = make_float4(acc[n][m][4], acc[n][m][5], acc[n][m][6], acc[n][m][7]);
            }
        }
    __syncthreads();
    // the warps: sums[0] holds the CTA's
    for (int i = threadIdx.x; i < MT * NW * COLS; i += kThreads) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += (&sums[w][0][0])[i];
        (&sums[0][0][0])[i] = v;
    }
    cluster.sync();
    // the cluster: each CTA finishes its share of the rows and columns
    for (int i = rank * kThreads + threadIdx.x; i < MT * COLS; i += ranks * kThreads) {
        const int m = i / COLS, c = i % COLS;
        float v[NW];
#pragma unroll
        for (int n = 0; n < NW; ++n) v[n] = 0.f;
        for (int r = 0; r < ranks; ++r) {
            const float* s = cluster.map_shared_rank(&sums[0][0][0], r);
#pragma unroll
            for (int n = 0; n < NW; ++n) v[n] += s[(n * MT + m) * COLS + c];
        }
        if (col0 + c < p.N) {
            if constexpr (LINEAR) {
                finish_linear(p, m, col0 + c, v[0]);
            } else if constexpr (NW == 1) {
                p.y[m * p.ldy + col0 + c] = __float2bfloat16_rn(v[0]);
            } else {
                glu::with_act(p.act, [&](auto act) {
                    float2 a, slope;
                    glu::act_value_slope<act.value>(make_float2(v[0], v[0]), a, slope);
                    p.y[m * p.ldy + col0 + c] = __float2bfloat16_rn(a.x * v[NW - 1]);
                });
                const int64_t at = m * p.ldg + col0 + c;
                if (p.g && p.keep32) {
                    static_cast<float*>(p.g)[at] = v[0];
                    static_cast<float*>(p.u)[at] = v[NW - 1];
                } else if (p.g) {
                    static_cast<__nv_bfloat16*>(p.g)[at] = __float2bfloat16_rn(v[0]);
                    static_cast<__nv_bfloat16*>(p.u)[at] = __float2bfloat16_rn(v[NW - 1]);
                }
            }
        }
    }
    cluster.sync();                        // nobody leaves while its sums may still be read
}

// The linear layer with W stored [N][K]: a warp takes kNkCols rows of W, lanes side by side along K, so that 2 kNkCols loads of 16
// bytes are in flight per thread.  SPLIT: the CTA's warps share one group of rows of W and deal K out among themselves (few
// columns), else each has its own.  Sums joined in a fixed order, as above.
constexpr int kNkCols = 4;
template <int MT, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 8) few_rows_nk_kernel(const FewParams p) {
    __shared__ float sums[SPLIT ? kWarps : 1][MT * kNkCols];
    constexpr int SHARE = SPLIT ? kWarps : 1;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t n0 = (SPLIT ? static_cast<int64_t>(blockIdx.x) : static_cast<int64_t>(blockIdx.x) * kWarps + warp) * kNkCols;
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
    float acc[MT][kNkCols] = {};
    if (n0 < p.N) {                        // N is a multiple of 8, and so of kNkCols
        constexpr int64_t STEP = 256 * SHARE;
        const __nv_bfloat16* const w = p.w0 + n0 * p.ldw;
        const auto take = [&](const uint4 (&wv)[kNkCols], const uint4 (&xv)[MT]) {
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const uint32_t xw[4] = {xv[m].x, xv[m].y, xv[m].z, xv[m].w};
#pragma unroll
                for (int c = 0; c < kNkCols; ++c) {
                    const uint32_t ww[4] = {wv[c].x, wv[c].y, wv[c].z, wv[c].w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[m][c] = fmaf(lo(xw[e]), lo(ww[e]), acc[m][c]);
                        acc[m][c] = fmaf(hi(xw[e]), hi(ww[e]), acc[m][c]);
                    }
                }
            }
        };
        const auto load = [&](int64_t k, uint4 (&wv)[kNkCols], uint4 (&xv)[MT]) {
#pragma unroll
            for (int c = 0; c < kNkCols; ++c) wv[c] = load_stream(w + c * p.ldw + k);
#pragma unroll
            for (int m = 0; m < MT; ++m) xv[m] = __ldg(reinterpret_cast<const uint4*>(p.x + m * p.ldx + k));
        };
        int64_t k = (SPLIT ? warp * 256 : 0) + lane * 8;
        for (; k + STEP < p.K; k += 2 * STEP) {
            uint4 w0[kNkCols], w1[kNkCols], x0[MT], x1[MT];
            load(k, w0, x0);
            load(k + STEP, w1, x1);
            take(w0, x0);
            take(w1, x1);
        }
        if (k < p.K) {
            uint4 w0[kNkCols], x0[MT];
            load(k, w0, x0);
            take(w0, x0);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int c = 0; c < kNkCols; ++c)
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) acc[m][c] += __shfl_xor_sync(0xFFFFFFFFu, acc[m][c], o);
    }
    float v = 0.f;                         // lane i has sum i
#pragma unroll
    for (int i = 0; i < MT * kNkCols; ++i)
        if (lane == i) v = acc[i / kNkCols][i % kNkCols];
    if constexpr (SPLIT) {
        if (lane < MT * kNkCols) sums[warp][lane] = v;
        __syncthreads();
        if (warp > 0) return;
        if (lane < MT * kNkCols)
#pragma unroll
            for (int i = 1; i < kWarps; ++i) v += sums[i][lane];
    }
    if (n0 < p.N && lane < MT * kNkCols) finish_linear(p, lane / kNkCols, n0 + lane % kNkCols, v);
}

// Columns per cluster and CTAs per cluster: all CTAs resident at once.  An SM draws its share of the memory's rate only with all
// its `per_sm` CTAs' loads in flight; with fewer CTAs each runs at the same pace, with more loads than that they share.  So
// the slowest SM, with ceil(CTAs / SMs) of them, takes max(that, per_sm) times a CTA's rounds.  64 columns where 32
// are not ahead by more than a twentieth (128-byte runs).
struct Deal {
    int cols, ranks;
};
Deal deal(int64_t K, int64_t N, int per_sm, int sms) {
    Deal best{64, 1};
    double least = 1e300;
    for (int cols = 64; cols >= 32; cols -= 32) {
        const int64_t blocks = atb::ceil_div(N, cols), rounds = atb::ceil_div(K, kWarps * (256 / cols) * 8);
        for (int ranks = 1; ranks <= 8 && ranks <= rounds; ++ranks) {
            const int64_t ctas = blocks * ranks;
            if (ranks > 1 && ctas > static_cast<int64_t>(per_sm) * sms) break;
            const double t = static_cast<double>(std::max<int64_t>(atb::ceil_div(ctas, sms), per_sm)) *
                             static_cast<double>(atb::ceil_div(rounds, ranks)) * (cols == 32 ? 1.05 : 1.0);
            if (t < least) { least = t; best = {cols, ranks}; }
        }
    }
    return best;
}

template <int MT, int NW, bool LINEAR>
cudaError_t launch(const FewParams& p, int sms, cudaStream_t stream) {
    const Deal d = deal(p.K, p.N, resident(MT, NW), sms);
    const unsigned grid = static_cast<unsigned>(atb::ceil_div(p.N, d.cols) * d.ranks), ranks = static_cast<unsigned>(d.ranks);
    return d.cols == 64 ? atb::launch_dependent(few_rows_kernel<MT, NW, 64, LINEAR>, grid, kThreads, ranks, 0, stream, p)
                        : atb::launch_dependent(few_rows_kernel<MT, NW, 32, LINEAR>, grid, kThreads, ranks, 0, stream, p);
}

template <int NW, bool LINEAR = false>
atb_status_t run(const FewParams& p, cudaStream_t stream) {
    int sms = 0;
    const atb_status_t s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    const cudaError_t e = p.M == 1 ? launch<1, NW, LINEAR>(p, sms, stream) : launch<2, NW, LINEAR>(p, sms, stream);
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "few-row product launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

}  // namespace

namespace atb {

atb_status_t few_rows_product(int64_t M, int64_t K, int64_t N, const void* X, int64_t ldx, const void* W, int64_t ldw, void* Y, int64_t ldy,
                              bool weights_settled, cudaStream_t stream) {
    FewParams p = {};
    p.M = static_cast<int>(M); p.K = K; p.N = N; p.ldx = ldx; p.ldw = ldw; p.ldy = ldy;
    p.x = static_cast<const __nv_bfloat16*>(X); p.w0 = static_cast<const __nv_bfloat16*>(W);
    p.y = static_cast<__nv_bfloat16*>(Y);
    p.weights_settled = weights_settled;
    return run<1>(p, stream);
}

atb_status_t few_rows_linear(const MmProblem& q, cudaStream_t stream) {
    FewParams p = {};
    p.M = static_cast<int>(q.M); p.K = q.K; p.N = q.N; p.ldx = q.A[0].ld; p.ldw = q.B[0].ld; p.ldy = q.ldc[0]; p.act = q.act;
    p.x = static_cast<const __nv_bfloat16*>(q.A[0].base); p.w0 = static_cast<const __nv_bfloat16*>(q.B[0].base);
    p.bias = q.bias; p.bias32 = q.bias32;
    p.r = q.R; p.ldr = q.ldr;
    p.out = q.C[0]; p.y32 = q.y32;
    p.z = q.C[1]; p.z32 = q.z32;
    if (q.layout == kMmNN) return run<1, true>(p, stream);
    int sms = 0;
    const atb_status_t s = op_device(&sms);
    if (s != ATB_OK) return s;
    // A group of 4 columns to a warp where those fill the SMs, else to a CTA, whose warps share K.  One row, K x N, warps and CTAs (us): 2048 x 5464
    // 7.8 and 8.0 (two rows 7.8 and 6.6), 1024 x 16384 7.7 and 7.9, 4096 x 10944 17.8 and 16.2, 10944 x 4096 30.6 and 15.7,
    // 4096 x 16384 23.6 and 22.2; from there on 2048 x 24576 18.0 and 17.9, 2048 x 32000 21.4 and 22.8, 4096 x 32000 40.9 and 39.5,
    // 1024 x 64000 21.5 and 23.5, 64 x 131072 11.5 and 35.7.
    const int64_t groups = ceil_div(q.N, kNkCols);
    const bool split = groups < static_cast<int64_t>(sms) * 8 * kWarps;
    const unsigned grid = static_cast<unsigned>(split ? groups : ceil_div(groups, kWarps));
    const auto go = [&](auto kernel) { return launch_dependent(kernel, grid, static_cast<unsigned>(kThreads), 1u, 0, stream, p); };
    const cudaError_t e = p.M == 1 ? (split ? go(few_rows_nk_kernel<1, true>) : go(few_rows_nk_kernel<1, false>))
                                   : (split ? go(few_rows_nk_kernel<2, true>) : go(few_rows_nk_kernel<2, false>));
    if (e != cudaSuccess) return fail(ATB_ERR_CUDA, "few-row linear launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

atb_status_t few_rows_glu(int64_t M, int64_t K, int64_t N, int act, const void* X, int64_t ldx, const void* Wg, const void* Wu, int64_t ldw, void* H,
                          void* G, void* U, bool keep32, cudaStream_t stream) {
    FewParams p = {};
    p.M = static_cast<int>(M); p.K = K; p.N = N; p.ldx = ldx; p.ldw = ldw; p.ldy = N; p.ldg = N; p.act = act;
    p.x = static_cast<const __nv_bfloat16*>(X);
    p.w0 = static_cast<const __nv_bfloat16*>(Wg); p.w1 = static_cast<const __nv_bfloat16*>(Wu);
    p.y = static_cast<__nv_bfloat16*>(H); p.g = G; p.u = U; p.keep32 = keep32;
    return run<2>(p, stream);
}

}  // namespace atb
