// Residual norm: the entry points of both directions, and the sums of its weights' gradients (sm_100a).  The row kernels are in
// residual_norm_forward.cuh and residual_norm_backward.cuh.
#include <algorithm>

#include "atb_residual_norm.cuh"

namespace residual_norm {
namespace {

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

// Walkers of the backward kernels: threads of a row and elements of a thread; none: the wide kernel.
struct Grid {
    int blocks, walkers;
};
// All that are resident, while each still has 4 rows, since its sums go through the workspace, but one per SM at least.
Grid grid_of(int64_t M, int64_t N) {
    const int w = width_of(N), per_block = w < kWidthCount && kWidths[w].threads == 32 ? 4 : 1, per_sm = w < kWidthCount ? blocks_of(kWidths[w].threads) : 2;
    const int64_t all = atb::ceil_div(M, per_block), most = static_cast<int64_t>(atb::kSmCount) * per_sm;
    int64_t blocks = atb::ceil_div(M, 4 * per_block);
    if (blocks < atb::kSmCount) blocks = atb::kSmCount;
    if (blocks > most) blocks = most;
    if (blocks > all) blocks = all;
    if (blocks < 1) blocks = 1;
    return {static_cast<int>(blocks), static_cast<int>(blocks) * per_block};
}
int walkers(int64_t M, int64_t N) { return grid_of(M, N).walkers; }

// The sums of walkers and columns -> the weights' gradients.  A block takes COLS columns: 32, or 8 where 32 would leave SMs without a block;
// its threads 512 / COLS walkers' sums of them at a time; then those in turn.  S0 = sum dz norm(h), S1 = sum dz, S2 = sum t norm(f) (or t f), S3 =
// sum t, where t is the gradient that arrives at h.
constexpr int kSumWarps = 16;
struct SumParams {
    const float* part;
    int walkers, post;
    int64_t N;
    Weights v;
    void *dw, *db, *dgate, *dpw, *dpb;
};
template <int COLS>
__global__ void __launch_bounds__(32 * kSumWarps) residual_norm_sum_kernel(const SumParams p) {
    constexpr int kSumRows = kSumWarps * 32 / COLS;
    __shared__ float s[kSumRows][4][COLS];
    const int c = threadIdx.x % COLS, first = threadIdx.x / COLS, sums = p.post ? 4 : 3;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * COLS + c;
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
    float v[4] = {};
    if (n < p.N) {
#pragma unroll 4
        for (int i = first; i < p.walkers; i += kSumRows) {
            const float* src = p.part + static_cast<int64_t>(i) * sums * p.N + n;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < sums) v[k] += src[k * p.N];
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) s[first][k][c] = v[k];
    __syncthreads();
    // a thread to a sum and column
    if (threadIdx.x < 4 * COLS) {
        float total = 0.f;
#pragma unroll 16
        for (int i = 0; i < kSumRows; ++i) total += s[i][threadIdx.x / COLS][c];
        s[0][threadIdx.x / COLS][c] = total;
    }
    __syncthreads();
    if (threadIdx.x >= COLS || n >= p.N) return;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = s[0][k][c];
    const auto weight = [&](const void* w, float none) {
        float o[1];
        if (p.v.w32) weights<float, 1>(w, static_cast<int>(n), none, o);
        else weights<__nv_bfloat16, 1>(w, static_cast<int>(n), none, o);
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
    const auto launch = w_type == ATB_F32 ? launch_forward_f32 : launch_forward_bf16;
    const cudaError_t e = launch(p, types_of(x_type, f_type), vec, post, st);
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
                          sums ? static_cast<float*>(workspace_dev) : nullptr, grid_of(M, N).blocks};
        const auto launch = w_type == ATB_F32 ? launch_backward_f32 : launch_backward_bf16;
        e = launch(p, types_of(x_type, f_type), vec, post, st);
    }
    if (e == cudaSuccess && sums) {
        const SumParams p{static_cast<const float*>(workspace_dev), M > 0 ? walkers(M, N) : 0, post, N, v, dW_dev, dB_dev, dgate_dev, dPW_dev, dPB_dev};
        e = N < 32 * atb::kSmCount ? atb::launch_dependent(residual_norm_sum_kernel<8>, static_cast<unsigned>(atb::ceil_div(N, 8)), 32u * kSumWarps, 1u, 0, st, p)
                                   : atb::launch_dependent(residual_norm_sum_kernel<32>, static_cast<unsigned>(atb::ceil_div(N, 32)), 32u * kSumWarps, 1u, 0, st, p);
    }
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "residual norm backward launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}
