// Linear layer with bias, activation and residual, forward and backward: the entry points, the gradient of the activation and the
// bias, and the order of the products.
//
//   z = x W + b, y = act(z) + r
//   dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum over rows of dz
//
// Forward: one launch - bias, activation and residual are the product's epilogue, on the FP32 accumulator.
// Backward: one pass over dy and z that writes dz (bf16: the tensor cores' operand) and sums it over the rows in FP32 before it
// is rounded, the sums of the blocks' rows, and one launch of the two products.  Where dz is dy (no activation, bf16) the pass
// only sums, and is left out where the bias has no gradient.
// The forward pass is bound by the product (8192 x 4096 x 10944 with z in FP32 504 us, 1.46 PFLOP/s) or, where rows are few, by W (16 rows,
// 2048 x 32000 stored [N][K]: 26.6 to 28.8 us, 4.6 to 5.0 TB/s; 250 tiles on 148 SMs, which take one or two); a prompt by launch, fill, one K loop
// and drain, 44 tiles on 74 pairs of SMs (509 x 2048 x 5464: 22 us, of which 18.5 are the product alone).  The gradient's pass is bound by memory: 8192 x 10944, z in FP32, 118 us (6.1 TB/s).  The two
// products after it run at 1.54 PFLOP/s alone (955 us) and slower under the power cap behind a forward pass.
#include <algorithm>

#include "atb_bf16_mm.h"
#include "atb_few_rows.h"
#include "dependent_launch.cuh"
#include "glu.cuh"

#include <cuda_bf16.h>

namespace {

bool known_type(int t) { return t == ATB_F32 || t == ATB_BF16; }
bool ld_ok(int64_t ld, int64_t least, int type) { return ld >= least && ld % (type == ATB_F32 ? 4 : 8) == 0; }

atb_status_t check_layer(int64_t M, int64_t K, int64_t N, int act, int w_layout, int y_type, int z_type, int bias_type) {
    if (act < ATB_ACT_SILU || act > ATB_ACT_NONE) return atb::fail(ATB_ERR_BAD_ARGUMENT, "act=%d: an atb_act_t, ATB_ACT_RELU or ATB_ACT_NONE", act);
    if (w_layout != ATB_W_KN && w_layout != ATB_W_NK) return atb::fail(ATB_ERR_BAD_ARGUMENT, "w_layout=%d: ATB_W_KN or ATB_W_NK", w_layout);
    if (!known_type(y_type) || !known_type(z_type) || !known_type(bias_type))
        return atb::fail(ATB_ERR_BAD_ARGUMENT, "y_type=%d, z_type=%d, bias_type=%d: ATB_F32 or ATB_BF16", y_type, z_type, bias_type);
    if (M < 0 || K < 8 || N < 8 || K % 8 != 0 || N % 8 != 0 || M > (1ll << 30) || K > (1ll << 30) || N > (1ll << 30))
        return atb::fail(ATB_ERR_BAD_SHAPE, "need M >= 0, K >= 8 and N >= 8 with K %% 8 == 0 and N %% 8 == 0 (got %lld, %lld, %lld)", (long long)M,
                         (long long)K, (long long)N);
    return ATB_OK;
}

// ---------------------------------------------------------------------------------- dz and its sums over the rows
struct GradParams {
    int64_t M, N, lddy;
    const void *dy, *z;
    __nv_bfloat16* dz;                     // [M][N], or NULL
    float* part;                           // [gridDim.y][N], or NULL
    int act;
};

constexpr int kGradWarps = 8, kGradThreads = kGradWarps * 32, kGradCols = 256;

template <bool FP32>
__device__ __forceinline__ void load8(const void* p, int64_t at, float (&v)[8]) {
    if constexpr (FP32) {
        const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
        const float4 a = __ldcs(s), b = __ldcs(s + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + at));
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(w[e] << 16);
            v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
        }
    }
}

// A block takes 256 columns (a lane 8 of them) and the rows blockIdx.y kGradWarps + warp, + gridDim.y kGradWarps, ...
template <bool Y32, bool Z32>
__global__ void __launch_bounds__(kGradThreads, 4) linear_grad_kernel(const GradParams p) {
    __shared__ float sums[kGradWarps][kGradCols];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * kGradCols + lane * 8;
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
    float sum[8] = {};
    if (n < p.N)                           // N is a multiple of 8
        glu::with_linear_act(p.act, [&](auto act) {
#pragma unroll 2
            for (int64_t m = static_cast<int64_t>(blockIdx.y) * kGradWarps + warp; m < p.M; m += static_cast<int64_t>(gridDim.y) * kGradWarps) {
                float d[8];
                load8<Y32>(p.dy, m * p.lddy + n, d);
                if constexpr (act.value != ATB_ACT_NONE) {
                    float z[8];
                    load8<Z32>(p.z, m * p.N + n, z);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float2 a, slope;
                        glu::linear_act<act.value>(make_float2(z[2 * e], z[2 * e + 1]), a, slope);
                        d[2 * e] *= slope.x;
                        d[2 * e + 1] *= slope.y;
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += d[e];
                if (p.dz) {
                    uint32_t o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const __nv_bfloat162 b2 = __floats2bfloat162_rn(d[2 * e], d[2 * e + 1]);
                        o[e] = *reinterpret_cast<const uint32_t*>(&b2);
                    }
                    *reinterpret_cast<uint4*>(p.dz + m * p.N + n) = make_uint4(o[0], o[1], o[2], o[3]);
                }
            }
        });
    if (!p.part) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[warp][lane * 8 + e] = sum[e];
    __syncthreads();
    const int c = threadIdx.x;
    float v = sums[0][c];
#pragma unroll
    for (int w = 1; w < kGradWarps; ++w) v += sums[w][c];
    const int64_t col = static_cast<int64_t>(blockIdx.x) * kGradCols + c;
    if (col < p.N) p.part[static_cast<int64_t>(blockIdx.y) * p.N + col] = v;
}

// db: the blocks' sums in their order, 32 columns per block, 8 warps that take every 8th.
__global__ void __launch_bounds__(256) linear_bias_kernel(const float* part, int parts, int64_t N, void* db, int db32) {
    __shared__ float s[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
    float v = 0.f;
    if (n < N) {
#pragma unroll 8
        for (int i = warp; i < parts; i += 8) v += part[static_cast<int64_t>(i) * N + n];
    }
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && n < N) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += s[i][lane];
        if (db32) static_cast<float*>(db)[n] = v;
        else static_cast<__nv_bfloat16*>(db)[n] = __float2bfloat16_rn(v);
    }
}

// Blocks along the rows: four blocks per SM in all, and no more, which would be a second round (8192 x 10944: 602 blocks for 592 places took
// 160 us); at least 4 rows for each warp.
int row_blocks(int64_t M, int64_t N) {
    const int64_t across = atb::ceil_div(N, kGradCols), most = atb::ceil_div(M, 4 * kGradWarps);
    int64_t blocks = 4 * atb::kSmCount / across;
    if (blocks > most) blocks = most;
    return static_cast<int>(blocks < 1 ? 1 : blocks);
}

size_t up256(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t dz_bytes(int64_t M, int64_t N) { return up256(2 * static_cast<size_t>(M) * static_cast<size_t>(N)); }
size_t part_bytes(int64_t M, int64_t N) { return up256(4 * static_cast<size_t>(row_blocks(M, N)) * static_cast<size_t>(N)); }

int products(atb::MmProblem* q, int64_t M, int64_t K, int64_t N, int w_layout, bool dx, bool dw) {
    int n = 0;
    if (dx) q[n++] = atb::mm_sizes(w_layout == ATB_W_KN ? atb::kMmNT : atb::kMmNN, atb::kMmStore, M, K, N);
    if (dw) q[n++] = w_layout == ATB_W_KN ? atb::mm_sizes(atb::kMmTN, atb::kMmStore, K, N, M) : atb::mm_sizes(atb::kMmTN, atb::kMmStore, N, K, M);
    return n;
}
// Sums of products that are split along K.
size_t split_bytes(int64_t M, int64_t K, int64_t N, int w_layout, bool dx, bool dw) {
    atb::MmProblem q[atb::kMmGroup];
    const int n = products(q, M, K, N, w_layout, dx, dw);
    return n ? atb::mm_partial_bytes(q, n) : 0;
}
// The workspace of a call, one area behind another: dz, where it is not dy and a product takes it; the blocks' sums, where the bias has a
// gradient; sums of split products.
struct Room {
    size_t dz, part, split;
    size_t all() const { return dz + part + split; }
};
Room room_of(int64_t M, int64_t K, int64_t N, int act, int y_type, int w_layout, bool dx, bool dw, bool db) {
    const bool is_dy = act == ATB_ACT_NONE && y_type == ATB_BF16;
    return {!is_dy && (dx || dw) ? dz_bytes(M, N) : 0, db ? part_bytes(M, N) : 0, split_bytes(M, K, N, w_layout, dx, dw)};
}

}  // namespace

extern "C" size_t atb_linear_workspace_bytes(int64_t M, int64_t K, int64_t N) {
    if (M <= atb::kFewRows || K < 1 || N < 1) return 0;
    const atb::MmProblem a = atb::mm_sizes(atb::kMmNN, atb::kMmLinear, M, N, K), b = atb::mm_sizes(atb::kMmNT, atb::kMmLinear, M, N, K);
    return std::max(atb::mm_partial_bytes(&a, 1), atb::mm_partial_bytes(&b, 1));
}

extern "C" atb_status_t atb_linear(int64_t M, int64_t K, int64_t N, int act, int y_type, const void* X_dev, int64_t ldx, int w_layout, const void* W_dev,
                                   int64_t ldw, int bias_type, const void* bias_dev, const void* R_dev, int64_t ldr, void* Y_dev, int64_t ldy,
                                   int z_type, void* Z_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    atb::clear_error();
    const atb_status_t s = check_layer(M, K, N, act, w_layout, y_type, z_type, bias_type);
    if (s != ATB_OK) return s;
    if (M == 0) return ATB_OK;
    if (!X_dev || !W_dev || !Y_dev) return atb::fail(ATB_ERR_NULL_POINTER, "X, W and Y must be non-NULL");
    const bool kn = w_layout == ATB_W_KN;
    if (!ld_ok(ldx, K, ATB_BF16) || !ld_ok(ldw, kn ? N : K, ATB_BF16) || !ld_ok(ldy, N, y_type) || (R_dev && !ld_ok(ldr, N, y_type)))
        return atb::fail(ATB_ERR_BAD_SHAPE, "ldx must be >= K, ldw >= %s, ldy and ldr >= N, multiples of 8 (FP32: of 4) (got %lld, %lld, %lld, %lld)", kn ? "N" : "K",
                         (long long)ldx, (long long)ldw, (long long)ldy, (long long)ldr);
    for (const void* p : {X_dev, W_dev, bias_dev, R_dev, (const void*)Y_dev, (const void*)Z_dev, (const void*)workspace_dev})
        if (!atb::aligned16(p)) return atb::fail(ATB_ERR_MISALIGNED, "all device pointers must be 16-byte aligned");
    const size_t need = atb_linear_workspace_bytes(M, K, N);
    if (need > 0 && !workspace_dev) return atb::fail(ATB_ERR_NULL_POINTER, "a workspace of %zu bytes is needed", need);
    if (workspace_bytes < need) return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
    atb::MmProblem q = atb::mm_sizes(kn ? atb::kMmNN : atb::kMmNT, atb::kMmLinear, M, N, K);
    q.act = act;
    q.A[0] = {X_dev, ldx}; q.B[0] = {W_dev, ldw};
    q.C[0] = Y_dev; q.ldc[0] = ldy;
    q.C[1] = Z_dev; q.ldc[1] = N;
    q.y32 = y_type == ATB_F32; q.z32 = z_type == ATB_F32; q.bias32 = bias_type == ATB_F32;
    q.bias = bias_dev;
    q.R = R_dev; q.ldr = ldr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // Up to two rows stream W once: 4096 x 10944 17.5 us (5.1 TB/s), where tensor cores, whose tiles take any number of rows up to 128, take 21
    // to 22 for three rows.
    return M <= atb::kFewRows ? atb::few_rows_linear(q, st) : atb::mm_launch(&q, 1, workspace_dev, st);
}

extern "C" size_t atb_linear_backward_workspace_bytes(int64_t M, int64_t K, int64_t N) {
    if (M < 1 || K < 1 || N < 1) return 0;
    size_t split = 0;                      // the largest of any choice of gradients and layout
    for (int wanted = 1; wanted < 4; ++wanted)
        for (const int layout : {ATB_W_KN, ATB_W_NK}) split = std::max(split, split_bytes(M, K, N, layout, wanted & 1, wanted & 2));
    return dz_bytes(M, N) + part_bytes(M, N) + split;
}
extern "C" size_t atb_linear_backward_call_workspace_bytes(int64_t M, int64_t K, int64_t N, int act, int y_type, int w_layout, int dX, int dW, int dbias) {
    return M < 1 || K < 1 || N < 1 ? 0 : room_of(M, K, N, act, y_type, w_layout, dX, dW, dbias).all();
}

extern "C" atb_status_t atb_linear_backward(int64_t M, int64_t K, int64_t N, int act, int y_type, const void* dY_dev, int64_t lddy, const void* X_dev,
                                            int64_t ldx, int w_layout, const void* W_dev, int64_t ldw, int z_type, const void* Z_dev, void* dX_dev,
                                            int64_t lddx, void* dW_dev, int64_t lddw, int bias_type, void* dbias_dev, void* workspace_dev,
                                            size_t workspace_bytes, void* stream) {
    atb::clear_error();
    atb_status_t s = check_layer(M, K, N, act, w_layout, y_type, z_type, bias_type);
    if (s != ATB_OK) return s;
    const bool kn = w_layout == ATB_W_KN;
    const int64_t w_rows = kn ? K : N, w_cols = kn ? N : K;
    const Room room = M > 0 ? room_of(M, K, N, act, y_type, w_layout, dX_dev, dW_dev, dbias_dev) : Room{};
    const size_t need = room.all();
    if (M > 0 && (!dY_dev || (!Z_dev && act != ATB_ACT_NONE) || (!X_dev && dW_dev) || (!W_dev && dX_dev) || (need > 0 && !workspace_dev)))
        return atb::fail(ATB_ERR_NULL_POINTER, "dY, Z (with an activation), X (for dW), W (for dX) and a workspace of %zu bytes must be non-NULL", need);
    if ((M > 0 && (!ld_ok(lddy, N, y_type) || (dW_dev && !ld_ok(ldx, K, ATB_BF16)) || (dX_dev && (!ld_ok(ldw, w_cols, ATB_BF16) || !ld_ok(lddx, K, ATB_BF16))))) ||
        (dW_dev && !ld_ok(lddw, w_cols, ATB_BF16)))
        return atb::fail(ATB_ERR_BAD_SHAPE, "lddy must be >= N, ldx and lddx >= K, ldw and lddw >= the columns that W is stored with, multiples of 8 (FP32: of 4)");
    for (const void* p : {dY_dev, X_dev, W_dev, Z_dev, (const void*)dX_dev, (const void*)dW_dev, (const void*)dbias_dev, (const void*)workspace_dev})
        if (!atb::aligned16(p)) return atb::fail(ATB_ERR_MISALIGNED, "all device pointers must be 16-byte aligned");
    if (workspace_bytes < need) return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int sms = 0;
    s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    if (M == 0) {          // no rows: the sums over them are 0
        cudaError_t e = cudaSuccess;
        if (dW_dev) e = cudaMemset2DAsync(dW_dev, lddw * 2, 0, w_cols * 2, w_rows, st);
        if (e == cudaSuccess && dbias_dev) e = cudaMemsetAsync(dbias_dev, 0, N * (bias_type == ATB_F32 ? 4 : 2), st);
        return e == cudaSuccess ? ATB_OK : atb::fail(ATB_ERR_CUDA, "cudaMemsetAsync: %s", cudaGetErrorString(e));
    }
    char* const area = static_cast<char*>(workspace_dev);
    atb::MmOperand dz = {dY_dev, lddy};
    if (room.dz > 0 || dbias_dev) {
        GradParams g = {};
        g.M = M; g.N = N; g.lddy = lddy;
        g.dy = dY_dev; g.z = Z_dev;
        g.act = act;
        const bool y32 = y_type == ATB_F32, z32 = z_type == ATB_F32;
        if (room.dz > 0) {
            g.dz = reinterpret_cast<__nv_bfloat16*>(area);
            dz = {area, N};
        }
        if (dbias_dev) g.part = reinterpret_cast<float*>(area + room.dz);
        const int parts = row_blocks(M, N);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(static_cast<unsigned>(atb::ceil_div(N, kGradCols)), static_cast<unsigned>(parts), 1);
        cfg.blockDim = dim3(kGradThreads, 1, 1);
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const auto kernel = y32 ? (z32 ? linear_grad_kernel<true, true> : linear_grad_kernel<true, false>)
                                : (z32 ? linear_grad_kernel<false, true> : linear_grad_kernel<false, false>);
        cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<const GradParams>(g));
        if (e == cudaSuccess && dbias_dev)
            e = atb::launch_dependent(linear_bias_kernel, static_cast<unsigned>(atb::ceil_div(N, 32)), 256u, 1u, 0, st, static_cast<const float*>(g.part), parts, N,
                                      dbias_dev, static_cast<int>(bias_type == ATB_F32));
        if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "linear gradient launch: %s", cudaGetErrorString(e));
    }
    atb::MmProblem q[atb::kMmGroup];
    const int n = products(q, M, K, N, w_layout, dX_dev, dW_dev);
    if (n == 0) return ATB_OK;
    atb::MmProblem* next = q;
    if (dX_dev) {
        atb::MmProblem& dx = *next++;
        dx.A[0] = dz; dx.B[0] = {W_dev, ldw};
        dx.C[0] = dX_dev; dx.ldc[0] = lddx;
    }
    if (dW_dev) {
        atb::MmProblem& dw = *next++;
        const atb::MmOperand x = {X_dev, ldx};
        dw.A[0] = kn ? x : dz; dw.B[0] = kn ? dz : x;
        dw.C[0] = dW_dev; dw.ldc[0] = lddw;
    }
    return atb::mm_launch(q, n, area + room.dz + room.part, st);
}
