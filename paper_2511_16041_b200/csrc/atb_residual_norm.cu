// Residual norm, forward (sm_100a), and the entry points of both directions: what joins a branch to the residual stream and norms it.
//
//   u = norm(f) pw + pb, or f;   h = scale x + gate u;   z = norm(h) w + b
//   norm(v) = (v - mean) r, r = 1 / sqrt(mean((v - mean)^2) + eps); rms: the mean is taken as 0
//
// Bound by memory: x and f are read and h and z written, once.  A row's threads hold at most 16 elements each, h stays in registers (FP32)
// between the two norms, so that z is made of the unrounded h.  Blocks stay and walk the rows; the next rows of x and f are
// on their way into shared memory (cp.async) meanwhile.  Sums as in the layer norm: around the warps' own means, joined in one exchange per
// norm.  Rows wider than the widest kernel are read again for every sum.
#include <algorithm>

#include "atb_residual_norm.cuh"

namespace residual_norm {
namespace {

constexpr int kThreads[] = {32, 64, 128, 256, 384, 512, 768, 1024};
template <class TX, class TF>
constexpr int kMostThreads = sizeof(TX) + sizeof(TF) == 8 ? 768 : 1024;        // two stages of rows in shared memory
template <class TX, class TF>
constexpr int kAhead = sizeof(TX) + sizeof(TF) == 4 ? 2 : 1;
// Blocks that stay on an SM: 1024 threads of 64 registers (768 an element at a time), 200 KB of rows.
__host__ __device__ constexpr int resident(int threads, int stage_bytes, bool vec) {
    const int by_threads = (vec ? 1024 : 768) / threads, by_room = 200 * 1024 / stage_bytes;
    const int most = by_threads < by_room ? by_threads : by_room;
    return most < 1 ? 1 : most;
}
template <class TX, class TF, int TPR, int NV, int VEC>
constexpr int kRoom = (kAhead<TX, TF> + 1) * static_cast<int>(RowSource<TX, VEC, TPR, NV>::STAGE_BYTES + RowSource<TF, VEC, TPR, NV>::STAGE_BYTES);

// Mean and 1 / spread of a row whose elements its threads hold in v; v becomes distances d, and norm(v) is d r + shift.
template <int TPR>
struct RowNorm {
    static constexpr int W = TPR / 32;
    int lane, warp, center;
    float elems, n, inv_n, inv_own, eps;
    template <int NV, int VEC>
    __device__ __forceinline__ void operator()(float (&v)[NV][VEC], const bool (&in)[NV], float2* red, float& mu, float& r, float& shift) const {
        float s[1] = {0.f}, mine = 0.f;
        if (center) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (in[i])
#pragma unroll
                    for (int e = 0; e < VEC; ++e) s[0] += v[i][e];
            warp_sum(s);
            mine = quotient(s[0], __shfl_sync(0xFFFFFFFFu, elems, warp), inv_own);       // the mean of the warp's elements
            s[0] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (in[i])
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    v[i][e] -= mine;
                    s[0] += v[i][e] * v[i][e];
                }
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

template <class TX, class TF, int VEC, int TPR, int NV, bool POST>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, resident(TPR == 32 ? 128 : TPR, kRoom<TX, TF, TPR, NV, VEC>, VEC > 1))
residual_norm_kernel(const FwdParams p) {
    using SX = RowSource<TX, VEC, TPR, NV>;
    using SF = RowSource<TF, VEC, TPR, NV>;
    using Shared = std::conditional_t<SX::SHARED, SX, SF>;
    constexpr int WALKERS = TPR == 32 ? 4 : 1, W = TPR / 32, AHEAD = kAhead<TX, TF>, STAGES = AHEAD + 1;
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
    bool in[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) in[i] = col + i * TPR * VEC < N;
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
        float v[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (in[i]) {
                Raw<TF, VEC> raw;
                sf.read(stage, m, i, raw);
                to_float(raw, v[i]);
            }
        float mu, r, shift;
        if constexpr (POST) {
            norm(v, in, red[0][turn], mu, r, shift);
            if (t == 0 && p.stats) { p.stats[2 * p.M + m] = mu; p.stats[3 * p.M + m] = r; }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (in[i]) {
                const int n = col + i * TPR * VEC;
                float a[VEC], b[VEC];
                if constexpr (POST) {
                    weights<VEC>(p.v.pw, p.v.w32, n, 1.f, a);
                    weights<VEC>(p.v.pb, p.v.w32, n, 0.f, b);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(fmaf(v[i][e], r, shift), a[e], b[e]);
                }
                Raw<TX, VEC> raw;
                sx.read(stage, m, i, raw);
                to_float(raw, b);
                weights<VEC>(p.v.gate, p.v.w32, n, 1.f, a);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(p.scale, b[e], a[e] * v[i][e]);
                store_f<TX, VEC>(static_cast<TX*>(p.h) + m * p.ldh + n, v[i]);
            }
        norm(v, in, red[1][turn], mu, r, shift);
        if (t == 0 && p.stats) { p.stats[m] = mu; p.stats[p.M + m] = r; }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (in[i]) {
                const int n = col + i * TPR * VEC;
                float a[VEC], b[VEC];
                weights<VEC>(p.v.w, p.v.w32, n, 1.f, a);
                weights<VEC>(p.v.b, p.v.w32, n, 0.f, b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(fmaf(v[i][e], r, shift), a[e], b[e]);
                store_f<TF, VEC>(static_cast<TF*>(p.z) + m * p.ldz + n, v[i]);
            }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
}

// Any width: x and f are read again for every sum.
template <class TX, class TF, int VEC, bool POST>
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
            weights<VEC>(p.v.pw, p.v.w32, n, 1.f, a);
            weights<VEC>(p.v.pb, p.v.w32, n, 0.f, b);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = fmaf((v[e] - fmu) * fr, a[e], b[e]);
        }
        load_f<TX, VEC>(x + n, b);
        weights<VEC>(p.v.gate, p.v.w32, n, 1.f, a);
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
        weights<VEC>(p.v.w, p.v.w32, n, 1.f, a);
        weights<VEC>(p.v.b, p.v.w32, n, 0.f, b);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = fmaf((v[e] - mu) * r, a[e], b[e]);
        store_f<TF, VEC>(static_cast<TF*>(p.z) + m * p.ldz + n, v);
    });
}

// ---------------------------------------------------------------------------------- host
template <class TX, class TF, int VEC, bool POST, int TPR>
cudaError_t launch_rows(const FwdParams& p, cudaStream_t st) {
    constexpr int NV = kElems / VEC, THREADS = TPR == 32 ? 128 : TPR, ROOM = kRoom<TX, TF, TPR, NV, VEC>;
    const int64_t all = atb::ceil_div(p.M, TPR == 32 ? 4 : 1), most = static_cast<int64_t>(atb::kSmCount) * resident(THREADS, ROOM, VEC > 1);
    return launch_ring(residual_norm_kernel<TX, TF, VEC, TPR, NV, POST>, static_cast<unsigned>(all < most ? all : most), THREADS, ROOM, st, p);
}
template <class TX, class TF, int VEC, bool POST>
cudaError_t launch(const FwdParams& p, cudaStream_t st) {
    for (const int t : kThreads) {
        if (t > kMostThreads<TX, TF> || p.N > static_cast<int64_t>(t) * kElems) continue;
        switch (t) {
            case 32: return launch_rows<TX, TF, VEC, POST, 32>(p, st);
            case 64: return launch_rows<TX, TF, VEC, POST, 64>(p, st);
            case 128: return launch_rows<TX, TF, VEC, POST, 128>(p, st);
            case 256: return launch_rows<TX, TF, VEC, POST, 256>(p, st);
            case 384: return launch_rows<TX, TF, VEC, POST, 384>(p, st);
            case 512: return launch_rows<TX, TF, VEC, POST, 512>(p, st);
            case 768: return launch_rows<TX, TF, VEC, POST, 768>(p, st);
            case 1024:
                if constexpr (kMostThreads<TX, TF> == 1024) return launch_rows<TX, TF, VEC, POST, 1024>(p, st);
        }
    }
    residual_norm_wide_kernel<TX, TF, VEC, POST><<<static_cast<unsigned>(p.M), 1024, 0, st>>>(p);
    return cudaGetLastError();
}
template <class TX, class TF>
cudaError_t launch_types(const FwdParams& p, bool vec, bool post, cudaStream_t st) {
    if (vec) return post ? launch<TX, TF, 8, true>(p, st) : launch<TX, TF, 8, false>(p, st);
    return post ? launch<TX, TF, 1, true>(p, st) : launch<TX, TF, 1, false>(p, st);
}

// ---------------------------------------------------------------------------------- checks
bool known_type(int t) { return t == ATB_F32 || t == ATB_BF16; }
int64_t size_of(int t) { return t == ATB_F32 ? 4 : 2; }
bool aligned_to(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }
bool vec_ok(const void* p, int64_t ld, int type) { return atb::aligned16(p) && ld * size_of(type) % 16 == 0; }

atb_status_t check_common(int64_t M, int64_t N, int kind, int x_type, int f_type, int w_type) {
    if (kind & ~(ATB_NORM_RMS | ATB_NORM_POST)) return atb::fail(ATB_ERR_BAD_ARGUMENT, "kind=%d: ATB_NORM_LAYER or ATB_NORM_RMS, with ATB_NORM_POST or without", kind);
    if (!known_type(x_type) || !known_type(f_type) || !known_type(w_type))
        return atb::fail(ATB_ERR_BAD_ARGUMENT, "x_type=%d, f_type=%d, w_type=%d: ATB_F32 or ATB_BF16", x_type, f_type, w_type);
    if (x_type == ATB_BF16 && f_type == ATB_F32) return atb::fail(ATB_ERR_BAD_ARGUMENT, "the branch's type is not wider than the stream's");
    if (M < 0 || N < 0 || M > 0x7FFFFFFFll - 32 || N > (1ll << 30))
        return atb::fail(ATB_ERR_BAD_SHAPE, "need 0 <= M < 2^31 - 32 and 0 <= N <= 2^30 (got %lld, %lld)", (long long)M, (long long)N);
    return ATB_OK;
}
Types types_of(int x_type, int f_type) { return x_type == ATB_BF16 ? kBf16 : f_type == ATB_BF16 ? kMixed : kF32; }

// The sums of walkers and columns -> the weights' gradients, 32 columns per block, 16 warps that take every 16th walker's sums, then the 16 in
// turn.  S0 = sum dz norm(h), S1 = sum dz, S2 = sum t norm(f) (or t f), S3 = sum t, where t is the gradient that arrives at h.
constexpr int kSumWarps = 16;
struct SumParams {
    const float* part;
    int walkers, post;
    int64_t N;
    Weights v;
    void *dw, *db, *dgate, *dpw, *dpb;
};
__global__ void __launch_bounds__(32 * kSumWarps) residual_norm_sum_kernel(const SumParams p) {
    __shared__ float s[kSumWarps][4][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sums = p.post ? 4 : 3;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
    float v[4] = {};
    if (n < p.N) {
#pragma unroll 4
        for (int i = warp; i < p.walkers; i += kSumWarps) {
            const float* src = p.part + static_cast<int64_t>(i) * sums * p.N + n;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < sums) v[k] += src[k * p.N];
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) s[warp][k][lane] = v[k];
    __syncthreads();
    if (warp != 0 || n >= p.N) return;
    for (int i = 1; i < kSumWarps; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += s[i][k][lane];
    const auto weight = [&](const void* w, float none) {
        float o[1];
        weights<1>(w, p.v.w32, static_cast<int>(n), none, o);
        return o[0];
    };
    const auto put = [&](void* out, float value) {
        if (!out) return;
        if (p.v.w32) static_cast<float*>(out)[n] = value;
        else static_cast<__nv_bfloat16*>(out)[n] = __float2bfloat16_rn(value);
    };
    put(p.dw, v[0]);
    put(p.db, v[1]);
    if (!p.post) {
        put(p.dgate, v[2]);
    } else {
        const float gate = weight(p.v.gate, 1.f);
        put(p.dgate, fmaf(weight(p.v.pw, 1.f), v[2], weight(p.v.pb, 0.f) * v[3]));
        put(p.dpw, gate * v[2]);
        put(p.dpb, gate * v[3]);
    }
}

}  // namespace
}  // namespace residual_norm

using namespace residual_norm;

extern "C" atb_status_t atb_residual_norm(int64_t M, int64_t N, int kind, int x_type, const void* X_dev, int64_t ldx, int f_type, const void* F_dev, int64_t ldf,
                                          float scale, int w_type, const void* gate_dev, const void* PW_dev, const void* PB_dev, const void* W_dev,
                                          const void* B_dev, float eps, void* H_dev, int64_t ldh, void* Z_dev, int64_t ldz, float* stats_dev, void* stream) {
    atb::clear_error();
    atb_status_t s = check_common(M, N, kind, x_type, f_type, w_type);
    if (s != ATB_OK) return s;
    if (!(eps >= 0.f)) return atb::fail(ATB_ERR_BAD_ARGUMENT, "eps must be >= 0");
    const bool post = kind & ATB_NORM_POST;
    if (!post && (PW_dev || PB_dev)) return atb::fail(ATB_ERR_BAD_ARGUMENT, "PW and PB belong to ATB_NORM_POST");
    if (M == 0 || N == 0) return ATB_OK;
    if (!X_dev || !F_dev || !H_dev || !Z_dev) return atb::fail(ATB_ERR_NULL_POINTER, "X, F, H and Z must be non-NULL");
    if (ldx < N || ldf < N || ldh < N || ldz < N)
        return atb::fail(ATB_ERR_BAD_SHAPE, "ldx=%lld, ldf=%lld, ldh=%lld and ldz=%lld must be >= N", (long long)ldx, (long long)ldf, (long long)ldh, (long long)ldz);
    if (!aligned_to(X_dev, size_of(x_type)) || !aligned_to(H_dev, size_of(x_type)) || !aligned_to(F_dev, size_of(f_type)) || !aligned_to(Z_dev, size_of(f_type)) ||
        !aligned_to(stats_dev, 4))
        return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements");
    bool vec = N % 8 == 0 && vec_ok(X_dev, ldx, x_type) && vec_ok(H_dev, ldh, x_type) && vec_ok(F_dev, ldf, f_type) && vec_ok(Z_dev, ldz, f_type);
    for (const void* w : {gate_dev, PW_dev, PB_dev, W_dev, B_dev}) {
        if (!aligned_to(w, size_of(w_type))) return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements");
        vec = vec && atb::aligned16(w);
    }
    int sms = 0;
    s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    const FwdParams p{M, N, ldx, ldf, ldh, ldz, X_dev, F_dev, {W_dev, B_dev, gate_dev, PW_dev, PB_dev, w_type == ATB_F32}, scale, eps, !(kind & ATB_NORM_RMS),
                      H_dev, Z_dev, stats_dev};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    switch (types_of(x_type, f_type)) {
        case kBf16: e = launch_types<__nv_bfloat16, __nv_bfloat16>(p, vec, post, st); break;
        case kMixed: e = launch_types<float, __nv_bfloat16>(p, vec, post, st); break;
        case kF32: e = launch_types<float, float>(p, vec, post, st); break;
    }
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "residual norm launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

extern "C" size_t atb_residual_norm_backward_workspace_bytes(int64_t M, int64_t N) {
    if (M < 1 || N < 1) return 0;
    return static_cast<size_t>(walkers(M, N)) * 4 * static_cast<size_t>(N) * sizeof(float);
}

extern "C" atb_status_t atb_residual_norm_backward(int64_t M, int64_t N, int kind, int x_type, const void* dZ_dev, int64_t lddz, const void* dH_dev, int64_t lddh,
                                                   const void* X_dev, int64_t ldx, int f_type, const void* F_dev, int64_t ldf, float scale, int w_type,
                                                   const void* gate_dev, const void* PW_dev, const void* PB_dev, const void* W_dev, const float* stats_dev,
                                                   void* dX_dev, int64_t lddx, void* dF_dev, int64_t lddf, void* dgate_dev, void* dPW_dev, void* dPB_dev,
                                                   void* dW_dev, void* dB_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    atb::clear_error();
    atb_status_t s = check_common(M, N, kind, x_type, f_type, w_type);
    if (s != ATB_OK) return s;
    const bool post = kind & ATB_NORM_POST;
    if (!post && (PW_dev || PB_dev || dPW_dev || dPB_dev)) return atb::fail(ATB_ERR_BAD_ARGUMENT, "PW, PB and their gradients belong to ATB_NORM_POST");
    if (N == 0) return ATB_OK;
    const bool sums = dgate_dev || dPW_dev || dPB_dev || dW_dev || dB_dev;
    if (M > 0 && (!dZ_dev || !X_dev || !F_dev || !stats_dev)) return atb::fail(ATB_ERR_NULL_POINTER, "dZ, X, F and the statistics must be non-NULL");
    if (M > 0 && sums && !workspace_dev) return atb::fail(ATB_ERR_NULL_POINTER, "the gradients of the weights need the workspace");
    if (M > 0 && (lddz < N || (dH_dev && lddh < N) || ldx < N || ldf < N || (dX_dev && lddx < N) || (dF_dev && lddf < N)))
        return atb::fail(ATB_ERR_BAD_SHAPE, "every leading dimension must be >= N");
    if (!aligned_to(X_dev, size_of(x_type)) || !aligned_to(dH_dev, size_of(x_type)) || !aligned_to(dX_dev, size_of(x_type)) || !aligned_to(F_dev, size_of(f_type)) ||
        !aligned_to(dZ_dev, size_of(f_type)) || !aligned_to(dF_dev, size_of(f_type)) || !aligned_to(stats_dev, 4) || !aligned_to(workspace_dev, 16))
        return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements, the workspace to 16 bytes");
    bool vec = N % 8 == 0 && vec_ok(X_dev, ldx, x_type) && vec_ok(F_dev, ldf, f_type) && vec_ok(dZ_dev, lddz, f_type) && (!dH_dev || vec_ok(dH_dev, lddh, x_type)) &&
               (!dX_dev || vec_ok(dX_dev, lddx, x_type)) && (!dF_dev || vec_ok(dF_dev, lddf, f_type));
    for (const void* w : {gate_dev, PW_dev, PB_dev, W_dev}) {
        if (!aligned_to(w, size_of(w_type))) return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements");
        vec = vec && atb::aligned16(w);
    }
    for (const void* w : {(const void*)dgate_dev, (const void*)dPW_dev, (const void*)dPB_dev, (const void*)dW_dev, (const void*)dB_dev})
        if (!aligned_to(w, size_of(w_type))) return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements");
    if (sums && workspace_bytes < atb_residual_norm_backward_workspace_bytes(M, N))
        return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, atb_residual_norm_backward_workspace_bytes(M, N));
    int sms = 0;
    s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    const Weights v{W_dev, nullptr, gate_dev, PW_dev, PB_dev, w_type == ATB_F32};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (M > 0 && (dX_dev || dF_dev || sums)) {
        const BwdParams p{M, N, lddz, lddh, ldx, ldf, lddx, lddf, dZ_dev, dH_dev, X_dev, F_dev, v, scale, !(kind & ATB_NORM_RMS), stats_dev, dX_dev, dF_dev,
                          sums ? static_cast<float*>(workspace_dev) : nullptr};
        e = launch_backward(p, types_of(x_type, f_type), vec, post, st);
    }
    if (e == cudaSuccess && sums) {
        const SumParams p{static_cast<const float*>(workspace_dev), M > 0 ? walkers(M, N) : 0, post, N, v, dW_dev, dB_dev, dgate_dev, dPW_dev, dPB_dev};
        e = atb::launch_dependent(residual_norm_sum_kernel, static_cast<unsigned>(atb::ceil_div(N, 32)), 32u * kSumWarps, 1u, 0, st, p);
    }
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "residual norm backward launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}
