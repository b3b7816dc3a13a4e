// Softmax cross entropy of a linear head without its logits, forward and backward.
//
//   l = x W^T, lse = log sum_v exp(l_v), loss = lse - l[label];  dl = (exp(l - lse) - [v = label]) dloss, dx = dl W, dW = dl^T x
//
// Forward: the logits of a tile stay in tensor memory; what leaves is, per row and group of columns, the maximum and
// the sum of exp(l - maximum), 8 bytes for 128 logits, and the label's logit.  A second kernel joins them.
// Backward: the logits are computed again, a piece of the vocabulary at a time; the epilogue turns them into dl, which
// the workspace holds for one piece (bf16: it is the operand of the next two products; in units of the largest dloss, see mm_unit).  dW of the piece is complete;
// dx is added up over the pieces in FP32, in their order, and rounded once.
// Tensor bound from a few hundred rows on: M = 8192, V = 131072, D = 4096 takes 25.6 to 27 ms for loss and gradients, 8 M V D operations
// at 1.30 to 1.37 PFLOP/s; the library product sustains 1.38 under the power cap.  M = 4096, V = 131072, D = 2048, loss
// alone, 1.62 to 1.66 ms, 1.32 to 1.36 PFLOP/s.  Computing the logits again costs a quarter of that; keeping them would take M x V numbers.
// A few rows are bound by reading W: 16 rows, V = 32000, D = 2048 28 us, 4.6 TB/s with both launches.
#include <cuda_bf16.h>

#include <algorithm>

#include "atb_bf16_mm.h"
#include "dependent_launch.cuh"

namespace {

// (maximum, sum of exp(x - maximum)) of two sets of numbers, of their union; an empty set is (-inf, 0).
__device__ __forceinline__ void join_stats(float& m, float& s, float m2, float s2) {
    const float top = fmaxf(m, m2), ref = top == -INFINITY ? 0.f : top;
    s = s * expf(m - ref) + s2 * expf(m2 - ref);
    m = top;
}

// One block per row: joins the row's pairs, in a fixed order.  Latency counts: a row's pairs are few, and where rows are few
// too this kernel is short of work; the loads of a thread are independent of one another.
constexpr int kJoinThreads = 128;
__global__ void __launch_bounds__(kJoinThreads) linear_ce_join_kernel(int64_t V, const float2* stats, int64_t per_row, const float* label_logit,
                                                                      const int64_t* labels, int64_t ignore_index, float* loss, float* lse) {
    __shared__ float2 part[kJoinThreads / 32];
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float m = -INFINITY, s = 0.f;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < per_row; i += kJoinThreads) {
        const float2 v = stats[row * per_row + i];
        join_stats(m, s, v.x, v.y);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) join_stats(m, s, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o));
    if (lane == 0) part[warp] = make_float2(m, s);
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < kJoinThreads / 32; ++w) join_stats(m, s, part[w].x, part[w].y);
        const int64_t label = labels[row];
        float z = m + logf(s), l = 0.f;
        if (label != ignore_index) {
            if (label < 0 || label >= V) z = l = __int_as_float(0x7FC00000);     // no such word: NaN, and so every gradient
            else l = z - label_logit[row];
        }
        lse[row] = z;
        loss[row] = l;
    }
}

__global__ void __launch_bounds__(256) linear_ce_round_kernel(const float* src, int64_t M, int64_t N, __nv_bfloat16* dst, int64_t ld) {
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
    const int64_t per_row = N / 8;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < M * per_row; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t m = i / per_row, n = (i - m * per_row) * 8;
        const float4 a = *reinterpret_cast<const float4*>(src + m * N + n), b = *reinterpret_cast<const float4*>(src + m * N + n + 4);
        __nv_bfloat162 o[4] = {__floats2bfloat162_rn(a.x, a.y), __floats2bfloat162_rn(a.z, a.w), __floats2bfloat162_rn(b.x, b.y),
                               __floats2bfloat162_rn(b.z, b.w)};
        *reinterpret_cast<uint4*>(dst + m * ld + n) = *reinterpret_cast<const uint4*>(o);
    }
}

atb_status_t check_head(int64_t M, int64_t V, int64_t D) {
    if (M < 0 || V < 1 || D < 8 || D % 8 != 0 || M > (1ll << 30) || V > (1ll << 30) || D > (1ll << 30))
        return atb::fail(ATB_ERR_BAD_SHAPE, "need M >= 0, V >= 1, D >= 8 with D %% 8 == 0 (got %lld, %lld, %lld)", (long long)M, (long long)V, (long long)D);
    return ATB_OK;
}
bool ld_ok(int64_t ld, int64_t least) { return ld >= least && ld % 8 == 0; }
size_t align256(size_t n) { return (n + 255) / 256 * 256; }

// Words of a piece: the caller's number rounded up to whole tiles, or (0) as many as keep dl within 512 MB, but at least 2048 (more for M
// above 131072).
int64_t piece_words(int64_t M, int64_t V, int64_t piece) {
    if (piece <= 0) {
        piece = (1ll << 28) / M / 256 * 256;
        if (piece < 2048) piece = 2048;
    }
    piece = atb::round_up(piece < V ? piece : V, 256);
    return piece;
}

// The products behind dl of a piece of n words, which are one launch: sizes and layouts of those wanted.
int gradient_products(atb::MmProblem* q, int64_t M, int64_t n, int64_t D, bool pieces, bool dx, bool dw) {
    int products = 0;
    if (dx) q[products++] = atb::mm_sizes(atb::kMmNN, pieces ? atb::kMmAccumulate : atb::kMmStore, M, D, n);
    if (dw) q[products++] = atb::mm_sizes(atb::kMmTN, atb::kMmStore, n, D, M);
    return products;
}

// The backward workspace: dl of a piece, FP32 sums of dx where there is more than one piece, the unit of dl, and the sums of a
// product that is split along K.
struct BackwardSpace {
    int64_t words;
    size_t sum, unit, partial, partial_bytes;      // offsets behind dl, size of the last part
};
BackwardSpace backward_space(int64_t M, int64_t V, int64_t D, int64_t piece) {
    BackwardSpace w;
    w.words = piece_words(M, V, piece);
    w.sum = align256(static_cast<size_t>(M) * static_cast<size_t>(w.words) * 2);
    w.unit = w.sum + (w.words < V ? align256(static_cast<size_t>(M) * static_cast<size_t>(D) * sizeof(float)) : 0);
    w.partial = w.unit + 256;
    // the last piece may be shorter than the others, with a plan of its own
    const int64_t first = V < w.words ? V : w.words, last = V - (V - 1) / w.words * w.words;
    w.partial_bytes = 0;
    for (const int64_t n : {first, last})
        for (int wanted = 1; wanted < 4; ++wanted) {
            atb::MmProblem q[atb::kMmGroup];
            const int products = gradient_products(q, M, n, D, w.words < V, wanted & 1, wanted & 2);
            w.partial_bytes = std::max(w.partial_bytes, atb::mm_partial_bytes(q, products));
        }
    return w;
}

}  // namespace

extern "C" size_t atb_linear_cross_entropy_workspace_bytes(int64_t M, int64_t V, int64_t D) {
    if (M < 1 || V < 1 || D < 1) return 0;
    return align256(static_cast<size_t>(M) * static_cast<size_t>(atb::mm_stats_per_row(M, V, D)) * sizeof(float2)) + static_cast<size_t>(M) * sizeof(float);
}

extern "C" atb_status_t atb_linear_cross_entropy(int64_t M, int64_t V, int64_t D, const void* X_dev, int64_t ldx, const void* W_dev, int64_t ldw,
                                                 const int64_t* labels_dev, int64_t ignore_index, float* loss_dev, float* lse_dev,
                                                 void* workspace_dev, size_t workspace_bytes, void* stream) {
    atb::clear_error();
    atb_status_t s = check_head(M, V, D);
    if (s != ATB_OK) return s;
    if (M == 0) return ATB_OK;
    if (!X_dev || !W_dev || !labels_dev || !loss_dev || !lse_dev || !workspace_dev)
        return atb::fail(ATB_ERR_NULL_POINTER, "all device pointers, including the workspace, must be non-NULL");
    if (!ld_ok(ldx, D) || !ld_ok(ldw, D))
        return atb::fail(ATB_ERR_BAD_SHAPE, "ldx=%lld and ldw=%lld must be >= D and multiples of 8", (long long)ldx, (long long)ldw);
    if (!atb::aligned16(X_dev) || !atb::aligned16(W_dev) || !atb::aligned16(workspace_dev) || (reinterpret_cast<uintptr_t>(labels_dev) & 7) ||
        (reinterpret_cast<uintptr_t>(loss_dev) & 3) || (reinterpret_cast<uintptr_t>(lse_dev) & 3))
        return atb::fail(ATB_ERR_MISALIGNED, "X, W and the workspace must be 16-byte aligned, labels, loss and lse to their elements");
    const size_t need = atb_linear_cross_entropy_workspace_bytes(M, V, D);
    if (workspace_bytes < need) return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    atb::MmProblem q;
    q.layout = atb::kMmNT; q.epilogue = atb::kMmRowStats;
    q.M = M; q.N = V; q.K = D;
    q.A[0] = {X_dev, ldx}; q.B[0] = {W_dev, ldw};
    q.labels = labels_dev;
    q.stats = static_cast<float2*>(workspace_dev);
    q.stats_ld = atb::mm_stats_per_row(M, V, D);
    q.label_logit = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + (need - static_cast<size_t>(M) * sizeof(float)));
    s = atb::mm_launch(&q, 1, nullptr, st);
    if (s != ATB_OK) return s;
    const cudaError_t e = atb::launch_dependent(linear_ce_join_kernel, static_cast<unsigned>(M), kJoinThreads, 1u, 0, st, V, static_cast<const float2*>(q.stats),
                                                q.stats_ld, static_cast<const float*>(q.label_logit), labels_dev, ignore_index, loss_dev, lse_dev);
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "linear cross entropy launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

extern "C" size_t atb_linear_cross_entropy_backward_workspace_bytes(int64_t M, int64_t V, int64_t D, int64_t piece) {
    if (M < 1 || V < 1 || D < 1) return 0;
    const BackwardSpace w = backward_space(M, V, D, piece);
    return w.partial + w.partial_bytes;
}

extern "C" atb_status_t atb_linear_cross_entropy_backward(int64_t M, int64_t V, int64_t D, const void* X_dev, int64_t ldx, const void* W_dev,
                                                          int64_t ldw, const int64_t* labels_dev, int64_t ignore_index, const float* lse_dev,
                                                          const float* dloss_dev, void* dX_dev, int64_t lddx, void* dW_dev, int64_t lddw,
                                                          int64_t piece, void* workspace_dev, size_t workspace_bytes, void* stream) {
    atb::clear_error();
    atb_status_t s = check_head(M, V, D);
    if (s != ATB_OK) return s;
    if (M > 0 && (!X_dev || !W_dev || !labels_dev || !lse_dev || !dloss_dev || !workspace_dev))
        return atb::fail(ATB_ERR_NULL_POINTER, "X, W, labels, lse, dloss and the workspace must be non-NULL");
    if (piece < 0) return atb::fail(ATB_ERR_BAD_ARGUMENT, "piece must be >= 0 (0: the library's choice)");
    if ((M > 0 && (!ld_ok(ldx, D) || !ld_ok(ldw, D) || (dX_dev && !ld_ok(lddx, D)))) || (dW_dev && !ld_ok(lddw, D)))
        return atb::fail(ATB_ERR_BAD_SHAPE, "ldx, ldw, lddx and lddw must be >= D and multiples of 8");
    if (!atb::aligned16(X_dev) || !atb::aligned16(W_dev) || !atb::aligned16(dX_dev) || !atb::aligned16(dW_dev) || !atb::aligned16(workspace_dev) ||
        (reinterpret_cast<uintptr_t>(labels_dev) & 7) || (reinterpret_cast<uintptr_t>(lse_dev) & 3) || (reinterpret_cast<uintptr_t>(dloss_dev) & 3))
        return atb::fail(ATB_ERR_MISALIGNED, "X, W, dX, dW and the workspace must be 16-byte aligned, labels, lse and dloss to their elements");
    const size_t need = atb_linear_cross_entropy_backward_workspace_bytes(M, V, D, piece);
    if (workspace_bytes < need) return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    if (M == 0) {
        const cudaError_t e = dW_dev ? cudaMemset2DAsync(dW_dev, lddw * 2, 0, D * 2, V, st) : cudaSuccess;
        return e == cudaSuccess ? ATB_OK : atb::fail(ATB_ERR_CUDA, "cudaMemset2DAsync: %s", cudaGetErrorString(e));
    }
    if (!dX_dev && !dW_dev) return ATB_OK;
    const BackwardSpace space = backward_space(M, V, D, piece);
    const int64_t words = space.words;
    uint16_t* const dl = static_cast<uint16_t*>(workspace_dev);
    float* const sum = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + space.sum);
    float* const unit = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + space.unit);
    void* const partial = static_cast<char*>(workspace_dev) + space.partial;
    for (int64_t v0 = 0; v0 < V; v0 += words) {
        const int64_t n = V - v0 < words ? V - v0 : words;
        const uint16_t* const Wv = static_cast<const uint16_t*>(W_dev) + v0 * ldw;
        atb::MmProblem q;
        q.layout = atb::kMmNT; q.epilogue = atb::kMmDlogits;
        q.M = M; q.N = n; q.K = D;
        q.A[0] = {X_dev, ldx}; q.B[0] = {Wv, ldw};
        q.C[0] = dl; q.ldc[0] = words;
        q.labels = labels_dev; q.ignore_index = ignore_index; q.col0 = v0;
        q.lse = lse_dev; q.scale = dloss_dev; q.unit = unit; q.first = v0 == 0;
        s = atb::mm_launch(&q, 1, nullptr, st);
        if (s != ATB_OK) return s;
        atb::MmProblem grad[atb::kMmGroup];
        const int products = gradient_products(grad, M, n, D, words < V, dX_dev, dW_dev);
        for (int j = 0; j < products; ++j) grad[j].factor = unit;
        if (dX_dev) {
            atb::MmProblem& dx = grad[0];
            dx.A[0] = {dl, words}; dx.B[0] = {Wv, ldw};
            dx.C32 = sum; dx.first = v0 == 0;
            dx.C[0] = dX_dev; dx.ldc[0] = lddx;
        }
        if (dW_dev) {
            atb::MmProblem& dw = grad[products - 1];
            dw.A[0] = {dl, words}; dw.B[0] = {X_dev, ldx};
            dw.C[0] = static_cast<uint16_t*>(dW_dev) + v0 * lddw; dw.ldc[0] = lddw;
        }
        s = atb::mm_launch(grad, products, partial, st);
        if (s != ATB_OK) return s;
    }
    cudaError_t e = cudaSuccess;
    if (dX_dev && words < V) {
        const int64_t vecs = M * (D / 8);
        const int blocks = static_cast<int>(atb::ceil_div(vecs, 256) < sms * 8 ? atb::ceil_div(vecs, 256) : sms * 8);
        e = atb::launch_dependent(linear_ce_round_kernel, static_cast<unsigned>(blocks), 256u, 1u, 0, st, static_cast<const float*>(sum), M, D,
                                  static_cast<__nv_bfloat16*>(dX_dev), lddx);
    }
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "linear cross entropy backward launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}
