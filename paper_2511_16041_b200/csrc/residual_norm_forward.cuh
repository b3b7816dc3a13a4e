// Residual norm, forward (sm_100a): what joins a branch to the residual stream and norms it.
//
//   u = norm(f) pw + pb, or f;   h = scale x + gate u;   z = norm(h) w + b
//   norm(v) = (v - mean) r, r = 1 / sqrt(mean((v - mean)^2) + eps); rms: the mean is taken as 0
//
// Bound by memory: x and f are read and h and z written, once.  A row's threads hold at most 16 elements each, h stays in registers (FP32)
// between the two norms, so that z is made of the unrounded h.  Blocks stay and walk the rows; the next rows of x and f are
// on their way into shared memory (cp.async) meanwhile.  Sums as in the layer norm: around the warps' own means, joined in one exchange per
// norm.  Rows wider than the widest kernel are read again for every sum.
// 16384 x 8192 with both norms and a gate 226 us at bf16 (4.8 TB/s), without the norm of f 176 us (6.1 TB/s); 8192 x 4096 bf16 45 us (6.0 TB/s), FP32 stream
// and bf16 branch 73; FP32 95.  The 512 threads of an SM issue in 45 to 55 % of the cycles; with both norms a row waits for two
// exchanges.
#pragma once
#include "atb_residual_norm.cuh"

namespace residual_norm {
namespace {

constexpr int kThreads[] = {32, 64, 96, 128, 192, 256, 384, 512, 768, 1024};
// The most that a kernel's predecessor takes: its rows are wider.
__host__ __device__ constexpr int fewer_of(int tpr) {
    int fewer = 0;
    for (const int t : kThreadCounts)
        if (t < tpr) fewer = t * kElems;
    return fewer;
}
template <class TX, class TF>
constexpr int kMostThreads = sizeof(TX) + sizeof(TF) == 8 ? 768 : 1024;        // two stages of rows in shared memory
// The vectors of weights stay in registers (a thread has the same columns of every row), but in the widest kernels, whose threads
// have too few, and but for FP32 gate pb, which would be one too many: it lies in shared memory (read again from the L1, which the rows on
// their way leave little of, 16384 x 8192 took 276 us).
__host__ __device__ constexpr bool keeps(int tpr) { return tpr <= 512; }
// Blocks that stay on an SM: 512 threads of 128 registers.
__host__ __device__ constexpr int resident(int tpr) { return tpr == 32 ? 4 : tpr >= 512 ? 1 : 512 / tpr; }
template <class TX, class TF, int TPR, int NV, int VEC>
constexpr int kStageBytes = static_cast<int>(RowSource<TX, VEC, TPR, NV>::STAGE_BYTES + RowSource<TF, VEC, TPR, NV>::STAGE_BYTES);
template <class TW, int TPR, int VEC, bool POST>
__host__ __device__ constexpr int c_bytes() { return keeps(TPR) && POST && !(sizeof(TW) == 2 && VEC == 8) ? kElems / 4 * (TPR == 32 ? 128 : TPR) * 16 : 0; }
// Rows on their way: 3, or what 200 KB per SM (with gate pb all 228 KB, of which a block takes 1 KB and its static arrays besides) hold beside the
// row in hand.
template <class TX, class TF, class TW, int TPR, int NV, int VEC, bool POST>
__host__ __device__ constexpr int ahead_of() {
    const int room = c_bytes<TW, TPR, VEC, POST>() ? 228 * 1024 / resident(TPR) - 1664 - c_bytes<TW, TPR, VEC, POST>() : 200 * 1024 / resident(TPR);
    const int stages = room / kStageBytes<TX, TF, TPR, NV, VEC>;
    return stages > 4 ? 3 : stages - 1;
}

// Mean and 1 / spread of a row whose elements its threads hold in v; v becomes distances d, and norm(v) is d r + shift.
template <int TPR>
struct RowNorm {
    static constexpr int W = TPR / 32;
    int lane, warp, center;
    float elems, n, inv_n, inv_own, eps;
    // Elements past the row's end: `in` tells (eights of single elements: by pairs' halves, eights of 8: whole eights)
    template <int CH, class In>
    __device__ __forceinline__ void operator()(float2 (&v)[CH][4], const In& in, float2* red, float& mu, float& r, float& shift) const {
        float s[1] = {0.f}, mine = 0.f;
        if (center) {
            float2 sum = both(0.f);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int k = 0; k < 4; ++k) sum = add2(sum, v[c][k]);      // 0 past the row's end
            s[0] = sum.x + sum.y;
            warp_sum(s);
            mine = quotient(s[0], __shfl_sync(0xFFFFFFFFu, elems, warp), inv_own);       // the mean of the warp's elements
        }
        float2 sq = both(0.f);
        const float2 from = both(-mine);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[c][k] = in.only(add2(v[c][k], from), c, k);
                sq = fma2(v[c][k], v[c][k], sq);
            }
        s[0] = sq.x + sq.y;
        warp_sum(s);
        mu = mine;
        if constexpr (TPR > 32) {
            if (lane == 0) red[warp] = make_float2(mine, s[0]);
            __syncthreads();
            const float2 part = lane < W ? red[lane] : make_float2(0.f, 0.f);
            if (center) {
                float sum[1] = {elems * part.x};
                warp_sum(sum);
                mu = quotient(sum[0], n, inv_n);
            }
            s[0] = part.y + elems * (part.x - mu) * (part.x - mu);
            warp_sum(s);
        }
        r = rsqrtf(s[0] * inv_n + eps);
        shift = (mine - mu) * r;
    }
};

// Which of a thread's elements are in the row.
template <int VEC, int TPR, int CH, int FULL>
struct Inside {
    using At = Eight<VEC, TPR, FULL>;
    bool in[CH][VEC == 8 ? 1 : 8];
    __device__ __forceinline__ Inside(int N, int col) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int g = 0; g < 8 / VEC; ++g) in[c][g] = At{N, col, c}.in(g);
    }
    __device__ __forceinline__ float2 only(float2 v, int c, int k) const {
        if constexpr (VEC == 8) return in[c][0] ? v : both(0.f);
        else return make_float2(in[c][(2 * k) % (8 / VEC)] ? v.x : 0.f, in[c][(2 * k + 1) % (8 / VEC)] ? v.y : 0.f);
    }
};

template <class TX, class TF, class TW, int VEC, int TPR, int NV, bool POST>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, resident(TPR)) residual_norm_kernel(const FwdParams p) {
    using SX = RowSource<TX, VEC, TPR, NV>;
    using SF = RowSource<TF, VEC, TPR, NV>;
    using Shared = std::conditional_t<SX::SHARED, SX, SF>;
    constexpr int WALKERS = TPR == 32 ? 4 : 1, W = TPR / 32, AHEAD = ahead_of<TX, TF, TW, TPR, NV, VEC, POST>(), STAGES = AHEAD + 1, CH = NV * VEC / 8;
    constexpr int FULL = full_of(TPR, NV, VEC, fewer_of(TPR));
    using At = Eight<VEC, TPR, FULL>;
    static_assert(AHEAD >= 1, "shared memory");
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float2 red[2][2][W];
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x, lane = threadIdx.x & 31;
    const int N = static_cast<int>(p.N), col = t * VEC;                 // group i: columns col + i TPR VEC ..
    const int64_t first = static_cast<int64_t>(blockIdx.x) * WALKERS + (TPR == 32 ? threadIdx.x >> 5 : 0), step = static_cast<int64_t>(gridDim.x) * WALKERS;
    const SX sx(sm100::smem_u32(ring), p.x, p.ldx, p.M, N, t);
    const SF sf(sm100::smem_u32(ring) + STAGES * SX::STAGE_BYTES, p.f, p.ldf, p.M, N, t);
    RowNorm<TPR> norm;
    {
        int count = 0;                     // elements of warp `lane`
#pragma unroll
        for (int i = 0; i < NV; ++i) count += max(0, min(32 * VEC, N - (i * TPR + lane * 32) * VEC));
        if (lane >= W) count = 0;
        norm.lane = lane;
        norm.warp = TPR == 32 ? 0 : threadIdx.x >> 5;
        norm.center = p.center;
        norm.elems = static_cast<float>(count);
        norm.n = static_cast<float>(N);
        norm.inv_n = 1.f / norm.n;
        norm.eps = p.eps;
        const int own = __shfl_sync(0xFFFFFFFFu, count, norm.warp);
        norm.inv_own = own > 0 ? 1.f / static_cast<float>(own) : 0.f;
    }
    const Inside<VEC, TPR, CH, FULL> in(N, col);
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
        if (first + s * step < p.M) {
            sx.fetch(s, first + s * step);
            sf.fetch(s, first + s * step);
        }
        async_commit();
    }
    // w, b, and a and c of h = scale x + a f + c (f: norm(f) with a norm of it, where a = gate pw and c = gate pb)
    constexpr int KEEP = keeps(TPR) ? kKept : kRead, KEEP_C = c_bytes<TW, TPR, VEC, POST>() ? kShared : keeps(TPR) && POST ? kKept : kRead;
    const Vector<TW, VEC, TPR, CH, FULL, KEEP> w_of(N, col, p.v.w, 1.f), b_of(N, col, p.v.b, 0.f);
    const Vector<TW, VEC, TPR, CH, FULL, KEEP, POST> a_of(N, col, p.v.gate, 1.f, p.v.pw, 1.f);
    const Vector<TW, VEC, TPR, CH, FULL, KEEP_C, true> c_of(N, col, POST ? p.v.gate : nullptr, 1.f, p.v.pb, 0.f,
                                                               sm100::smem_u32(ring) + STAGES * kStageBytes<TX, TF, TPR, NV, VEC>);
    const float2 scale = both(p.scale);
    int stage = 0, turn = 0;
    for (int64_t m = first; m < p.M; m += step, turn ^= 1) {
        const int ahead = stage == 0 ? AHEAD : stage - 1;               // the stage that the row before this one has left
        if (m + AHEAD * step < p.M) {
            sx.fetch(ahead, m + AHEAD * step);
            sf.fetch(ahead, m + AHEAD * step);
        }
        async_commit();
        async_wait<AHEAD>();
        row_barrier<Shared, VEC, TPR>();
        float2 v[CH][4];
#pragma unroll
        for (int c = 0; c < CH; ++c) At{N, col, c}.template read<TF>(sf, stage, m, v[c]);
        float mu, r, shift;
        if constexpr (POST) {
            norm(v, in, red[0][turn], mu, r, shift);
            if (t == 0 && p.stats) { p.stats[2 * p.M + m] = mu; p.stats[3 * p.M + m] = r; }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const At at{N, col, c};
            float2 a[4], x[4];
            at.template read<TX>(sx, stage, m, x);
            a_of.get(at, a);
            if constexpr (POST) {
                float2 c_[4];
                c_of.get(at, c_);
                const float2 r2 = both(r), shift2 = both(shift);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[c][k] = fma2(fma2(v[c][k], r2, shift2), a[k], c_[k]);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) v[c][k] = mul2(v[c][k], a[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) v[c][k] = in.only(fma2(scale, x[k], v[c][k]), c, k);
            at.template store<TX>(static_cast<TX*>(p.h) + m * p.ldh, v[c]);
        }
        norm(v, in, red[1][turn], mu, r, shift);
        if (t == 0 && p.stats) { p.stats[m] = mu; p.stats[p.M + m] = r; }
        const float2 r2 = both(r), shift2 = both(shift);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const At at{N, col, c};
            float2 a[4], b[4];
            w_of.get(at, a);
            b_of.get(at, b);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[c][k] = fma2(fma2(v[c][k], r2, shift2), a[k], b[k]);
            at.template store<TF>(static_cast<TF*>(p.z) + m * p.ldz, v[c]);
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
}

// Any width: x and f are read again for every sum.
template <class TX, class TF, class TW, int VEC, bool POST>
__global__ void __launch_bounds__(1024) residual_norm_wide_kernel(const FwdParams p) {
    __shared__ float red[4][32][1];
    const int64_t m = blockIdx.x;
    const TX* x = static_cast<const TX*>(p.x) + m * p.ldx;
    const TF* f = static_cast<const TF*>(p.f) + m * p.ldf;
    const float n_all = static_cast<float>(p.N), inv_n = 1.f / n_all;
    float fmu = 0.f, fr = 1.f, mu = 0.f, s[1] = {0.f}, v[VEC], a[VEC];
    const auto each = [&](auto&& body) {
        for (int64_t n = threadIdx.x * VEC; n < p.N; n += 1024 * VEC) body(static_cast<int>(n));
    };
    if constexpr (POST) {
        if (p.center) {
            each([&](int n) {
                load_f<TF, VEC>(f + n, v);
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[0] += v[e];
            });
            row_sum<1024, 1>(s, red[0]);
            fmu = quotient(s[0], n_all, inv_n);
            s[0] = 0.f;
        }
        each([&](int n) {
            load_f<TF, VEC>(f + n, v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[0] += (v[e] - fmu) * (v[e] - fmu);
        });
        row_sum<1024, 1>(s, red[1]);
        fr = rsqrtf(s[0] * inv_n + p.eps);
        s[0] = 0.f;
        if (threadIdx.x == 0 && p.stats) { p.stats[2 * p.M + m] = fmu; p.stats[3 * p.M + m] = fr; }
    }
    const auto h_of = [&](int n) {
        float b[VEC];
        load_f<TF, VEC>(f + n, v);
        if constexpr (POST) {
            weights<TW, VEC>(p.v.pw, n, 1.f, a);
            weights<TW, VEC>(p.v.pb, n, 0.f, b);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = fmaf((v[e] - fmu) * fr, a[e], b[e]);
        }
        load_f<TX, VEC>(x + n, b);
        weights<TW, VEC>(p.v.gate, n, 1.f, a);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = fmaf(p.scale, b[e], a[e] * v[e]);
    };
    if (p.center) {
        each([&](int n) {
            h_of(n);
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[0] += v[e];
        });
        row_sum<1024, 1>(s, red[2]);
        mu = quotient(s[0], n_all, inv_n);
        s[0] = 0.f;
    }
    each([&](int n) {
        h_of(n);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[0] += (v[e] - mu) * (v[e] - mu);
    });
    row_sum<1024, 1>(s, red[3]);
    const float r = rsqrtf(s[0] * inv_n + p.eps);
    if (threadIdx.x == 0 && p.stats) { p.stats[m] = mu; p.stats[p.M + m] = r; }
    each([&](int n) {
        float b[VEC];
        h_of(n);
        store_f<TX, VEC>(static_cast<TX*>(p.h) + m * p.ldh + n, v);
        weights<TW, VEC>(p.v.w, n, 1.f, a);
        weights<TW, VEC>(p.v.b, n, 0.f, b);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = fmaf((v[e] - mu) * r, a[e], b[e]);
        store_f<TF, VEC>(static_cast<TF*>(p.z) + m * p.ldz + n, v);
    });
}

// ---------------------------------------------------------------------------------- host
template <class TX, class TF, class TW, int VEC, bool POST, int TPR>
cudaError_t launch_rows(const FwdParams& p, cudaStream_t st) {
    constexpr int NV = kElems / VEC, THREADS = TPR == 32 ? 128 : TPR, ROOM = (ahead_of<TX, TF, TW, TPR, NV, VEC, POST>() + 1) * kStageBytes<TX, TF, TPR, NV, VEC> + c_bytes<TW, TPR, VEC, POST>();
    const int64_t all = atb::ceil_div(p.M, TPR == 32 ? 4 : 1), most = static_cast<int64_t>(atb::kSmCount) * resident(TPR);
    return launch_ring<&residual_norm_kernel<TX, TF, TW, VEC, TPR, NV, POST>>(static_cast<unsigned>(all < most ? all : most), THREADS, ROOM, st, p);
}
template <class TX, class TF, class TW, int VEC, bool POST>
cudaError_t launch(const FwdParams& p, cudaStream_t st) {
    for (const int t : kThreads) {
        if (t > kMostThreads<TX, TF> || p.N > static_cast<int64_t>(t) * kElems) continue;
        switch (t) {
            case 32: return launch_rows<TX, TF, TW, VEC, POST, 32>(p, st);
            case 64: return launch_rows<TX, TF, TW, VEC, POST, 64>(p, st);
            case 96: return launch_rows<TX, TF, TW, VEC, POST, 96>(p, st);
            case 128: return launch_rows<TX, TF, TW, VEC, POST, 128>(p, st);
            case 192: return launch_rows<TX, TF, TW, VEC, POST, 192>(p, st);
            case 256: return launch_rows<TX, TF, TW, VEC, POST, 256>(p, st);
            case 384: return launch_rows<TX, TF, TW, VEC, POST, 384>(p, st);
            case 512: return launch_rows<TX, TF, TW, VEC, POST, 512>(p, st);
            case 768: return launch_rows<TX, TF, TW, VEC, POST, 768>(p, st);
            case 1024:
                if constexpr (kMostThreads<TX, TF> == 1024) return launch_rows<TX, TF, TW, VEC, POST, 1024>(p, st);
        }
    }
    residual_norm_wide_kernel<TX, TF, TW, VEC, POST><<<static_cast<unsigned>(p.M), 1024, 0, st>>>(p);
    return cudaGetLastError();
}
template <class TX, class TF, class TW>
cudaError_t launch_types(const FwdParams& p, bool vec, bool post, cudaStream_t st) {
    if (vec) return post ? launch<TX, TF, TW, 8, true>(p, st) : launch<TX, TF, TW, 8, false>(p, st);
    return post ? launch<TX, TF, TW, 1, true>(p, st) : launch<TX, TF, TW, 1, false>(p, st);
}

template <class TW>
cudaError_t launch_forward(const FwdParams& p, Types types, bool vec, bool post, cudaStream_t st) {
    switch (types) {
        case kBf16: return launch_types<__nv_bfloat16, __nv_bfloat16, TW>(p, vec, post, st);
        case kMixed: return launch_types<float, __nv_bfloat16, TW>(p, vec, post, st);
        default: return launch_types<float, float, TW>(p, vec, post, st);
    }
}

}  // namespace
}  // namespace residual_norm
