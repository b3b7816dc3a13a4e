// Gated feed-forward block, forward and backward: the entry points and the order of the products.
//
//   g = x Wg, u = x Wu, h = act(g) u, y = h Wd
//   dh = dy Wd^T, du = dh act(g), dg = dh u act'(g), dx = dg Wg^T + du Wu^T, dWg = x^T dg, dWu = x^T du, dWd = h^T dy
//
// Forward: one kernel for both projections, the activation and the product (x is loaded once for both), one for y.
// Backward: dh never reaches memory - the epilogue of its product turns it into dg and du; the two products
// behind dx are one walk over 2 F, and dx and the three weight gradients are one launch.  h, dg and du are bf16 between the products: they
// are operands of the tensor cores, which take bf16; the rounding costs 2^-9 of the value.  g and u, which no product takes, are kept
// as the caller asks: FP32, or bf16 at half the memory (one rounding more in dx, dWg, dWu: 0.0030 of their norm off instead of 0.0024).
#include <algorithm>

#include "atb_bf16_mm.h"
#include "atb_few_rows.h"

namespace {

struct Block {
    int64_t M, D, F;
    int act;                               // without ATB_KEEP_F32
};

atb_status_t check_block(const Block& b) {
    if (b.act != ATB_ACT_SILU && b.act != ATB_ACT_GELU && b.act != ATB_ACT_GELU_TANH)
        return atb::fail(ATB_ERR_BAD_ARGUMENT, "act=%d: ATB_ACT_SILU, ATB_ACT_GELU or ATB_ACT_GELU_TANH", b.act);
    if (b.M < 0 || b.D < 8 || b.F < 8 || b.D % 8 != 0 || b.F % 8 != 0 || b.M > (1ll << 30) || b.D > (1ll << 30) || b.F > (1ll << 30))
        return atb::fail(ATB_ERR_BAD_SHAPE, "need M >= 0, D >= 8 and F >= 8 with D %% 8 == 0 and F %% 8 == 0 (got %lld, %lld, %lld)", (long long)b.M,
                         (long long)b.D, (long long)b.F);
    return ATB_OK;
}
bool ld_ok(int64_t ld, int64_t least) { return ld >= least && ld % 8 == 0; }
// dg and du in the workspace, [M][F] bf16 each, up to the next 256 bytes.
size_t glu_gradient_bytes(int64_t M, int64_t F) { return (4 * static_cast<size_t>(M) * static_cast<size_t>(F) + 255) / 256 * 256; }

// The products behind dh, which are one launch: sizes and layouts of those wanted.
int gradient_products(atb::MmProblem* q, int64_t M, int64_t D, int64_t F, bool dx, bool dw, bool dwd) {
    int n = 0;
    if (dx) q[n++] = atb::mm_sizes(atb::kMmNT, atb::kMmStore, M, D, F, 2, 1);
    if (dw) q[n++] = atb::mm_sizes(atb::kMmTN, atb::kMmStore, D, F, M, 1, 2);
    if (dwd) q[n++] = atb::mm_sizes(atb::kMmTN, atb::kMmStore, F, D, M);
    return n;
}
// Workspace of the gradients wanted: dg and du, and the sums of products that are split along K.
size_t gradient_bytes(int64_t M, int64_t D, int64_t F, bool dx, bool dw, bool dwd) {
    atb::MmProblem q[atb::kMmGroup];
    const atb::MmProblem dh = atb::mm_sizes(atb::kMmNT, atb::kMmGluBackward, M, F, D);
    const int n = gradient_products(q, M, D, F, dx, dw, dwd);
    return glu_gradient_bytes(M, F) + std::max(atb::mm_partial_bytes(&dh, 1), n ? atb::mm_partial_bytes(q, n) : 0);
}

}  // namespace

extern "C" size_t atb_gated_ffn_workspace_bytes(int64_t M, int64_t D, int64_t F) {
    if (M <= atb::kFewRows || D < 1 || F < 1) return 0;
    // the sums of a product that is split along K; the two products take turns
    const atb::MmProblem up = atb::mm_sizes(atb::kMmNN, atb::kMmGlu, M, F, D), down = atb::mm_sizes(atb::kMmNN, atb::kMmStore, M, D, F);
    return std::max(atb::mm_partial_bytes(&up, 1), atb::mm_partial_bytes(&down, 1));
}

extern "C" atb_status_t atb_gated_ffn(int64_t M, int64_t D, int64_t F, int act, const void* X_dev, int64_t ldx, const void* Wg_dev,
                                      const void* Wu_dev, int64_t ldw, const void* Wd_dev, int64_t ldwd, void* Y_dev, int64_t ldy,
                                      void* H_dev, void* G_dev, void* U_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    atb::clear_error();
    const bool keep32 = act >= 0 && (act & ATB_KEEP_F32);
    if (keep32) act &= ~ATB_KEEP_F32;
    atb_status_t s = check_block({M, D, F, act});
    if (s != ATB_OK) return s;
    if (M == 0) return ATB_OK;
    if (!X_dev || !Wg_dev || !Wu_dev || !Wd_dev || !Y_dev || !H_dev || !G_dev != !U_dev)
        return atb::fail(ATB_ERR_NULL_POINTER, "X, Wg, Wu, Wd, Y and H must be non-NULL, G and U both or neither");
    if (!ld_ok(ldx, D) || !ld_ok(ldw, F) || !ld_ok(ldwd, D) || !ld_ok(ldy, D))
        return atb::fail(ATB_ERR_BAD_SHAPE, "ldx, ldwd and ldy must be >= D, ldw >= F, all multiples of 8 (got %lld, %lld, %lld, %lld)", (long long)ldx,
                         (long long)ldwd, (long long)ldy, (long long)ldw);
    for (const void* p : {X_dev, Wg_dev, Wu_dev, Wd_dev, (const void*)Y_dev, (const void*)H_dev, (const void*)G_dev, (const void*)U_dev, (const void*)workspace_dev})
        if (!atb::aligned16(p)) return atb::fail(ATB_ERR_MISALIGNED, "all device pointers must be 16-byte aligned");
    const size_t need = atb_gated_ffn_workspace_bytes(M, D, F);
    if (need > 0 && !workspace_dev) return atb::fail(ATB_ERR_NULL_POINTER, "a workspace of %zu bytes is needed", need);
    if (workspace_bytes < need) return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
    cudaStream_t st = static_cast<cudaStream_t>(stream);

    if (M <= atb::kFewRows) {
        s = atb::few_rows_glu(M, D, F, act, X_dev, ldx, Wg_dev, Wu_dev, ldw, H_dev, G_dev, U_dev, keep32, st);
        return s != ATB_OK ? s : atb::few_rows_product(M, F, D, H_dev, F, Wd_dev, ldwd, Y_dev, ldy, true, st);
    }
    atb::MmProblem up;
    up.layout = atb::kMmNN; up.epilogue = atb::kMmGlu;
    up.M = M; up.N = F; up.K = D; up.act = act; up.keep32 = keep32 && G_dev;
    up.A[0] = {X_dev, ldx}; up.B[0] = {Wg_dev, ldw}; up.B[1] = {Wu_dev, ldw};
    up.C[0] = H_dev; up.C[1] = G_dev; up.C[2] = U_dev;
    up.ldc[0] = up.ldc[1] = up.ldc[2] = F;
    s = atb::mm_launch(&up, 1, workspace_dev, st);
    if (s != ATB_OK) return s;

    atb::MmProblem down;
    down.layout = atb::kMmNN; down.epilogue = atb::kMmStore;
    down.M = M; down.N = D; down.K = F;
    down.A[0] = {H_dev, F}; down.B[0] = {Wd_dev, ldwd};
    down.C[0] = Y_dev; down.ldc[0] = ldy;
    return atb::mm_launch(&down, 1, workspace_dev, st);
}

extern "C" size_t atb_gated_ffn_backward_workspace_bytes(int64_t M, int64_t D, int64_t F) {
    if (M < 1 || D < 1 || F < 1) return 0;
    size_t need = 0;                       // the largest of any choice of gradients
    for (int wanted = 1; wanted < 8; ++wanted) need = std::max(need, gradient_bytes(M, D, F, wanted & 1, wanted & 2, wanted & 4));
    return need;
}

extern "C" atb_status_t atb_gated_ffn_backward(int64_t M, int64_t D, int64_t F, int act, const void* dY_dev, int64_t lddy, const void* X_dev,
                                               int64_t ldx, const void* Wg_dev, const void* Wu_dev, int64_t ldw, const void* Wd_dev, int64_t ldwd,
                                               const void* H_dev, const void* G_dev, const void* U_dev, void* dX_dev, int64_t lddx, void* dWg_dev,
                                               void* dWu_dev, int64_t lddw, void* dWd_dev, int64_t lddwd, void* workspace_dev,
                                               size_t workspace_bytes, void* stream) {
    atb::clear_error();
    const bool keep32 = act >= 0 && (act & ATB_KEEP_F32);
    if (keep32) act &= ~ATB_KEEP_F32;
    atb_status_t s = check_block({M, D, F, act});
    if (s != ATB_OK) return s;
    if (!dWg_dev != !dWu_dev) return atb::fail(ATB_ERR_NULL_POINTER, "dWg and dWu are written both or neither");
    if (M > 0 && (!dY_dev || !X_dev || !Wg_dev || !Wu_dev || !Wd_dev || !H_dev || !G_dev || !U_dev || !workspace_dev))
        return atb::fail(ATB_ERR_NULL_POINTER, "dY, X, the weights, H, G, U and the workspace must be non-NULL");
    if ((M > 0 && (!ld_ok(lddy, D) || !ld_ok(ldx, D) || !ld_ok(ldw, F) || !ld_ok(ldwd, D))) || (dX_dev && M > 0 && !ld_ok(lddx, D)) ||
        (dWg_dev && !ld_ok(lddw, F)) || (dWd_dev && !ld_ok(lddwd, D)))
        return atb::fail(ATB_ERR_BAD_SHAPE, "lddy, ldx, ldwd, lddx and lddwd must be >= D, ldw and lddw >= F, all multiples of 8");
    for (const void* p : {dY_dev, X_dev, Wg_dev, Wu_dev, Wd_dev, H_dev, G_dev, U_dev, (const void*)dX_dev, (const void*)dWg_dev, (const void*)dWu_dev,
                          (const void*)dWd_dev, (const void*)workspace_dev})
        if (!atb::aligned16(p)) return atb::fail(ATB_ERR_MISALIGNED, "all device pointers must be 16-byte aligned");
    const size_t need = M > 0 ? gradient_bytes(M, D, F, dX_dev, dWg_dev, dWd_dev) : 0;
    if (workspace_bytes < need) return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes, need);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (M == 0) {          // no rows: the sums over them are 0
        int sms = 0;
        s = atb::op_device(&sms);
        if (s != ATB_OK) return s;
        cudaError_t e = cudaSuccess;
        if (dWg_dev) e = cudaMemset2DAsync(dWg_dev, lddw * 2, 0, F * 2, D, st);
        if (e == cudaSuccess && dWu_dev) e = cudaMemset2DAsync(dWu_dev, lddw * 2, 0, F * 2, D, st);
        if (e == cudaSuccess && dWd_dev) e = cudaMemset2DAsync(dWd_dev, lddwd * 2, 0, D * 2, F, st);
        return e == cudaSuccess ? ATB_OK : atb::fail(ATB_ERR_CUDA, "cudaMemset2DAsync: %s", cudaGetErrorString(e));
    }
    uint16_t* const dG = static_cast<uint16_t*>(workspace_dev);
    uint16_t* const dU = dG + M * F;
    void* const partial = static_cast<char*>(workspace_dev) + glu_gradient_bytes(M, F);

    if (dX_dev || dWg_dev) {
        atb::MmProblem dh;
        dh.layout = atb::kMmNT; dh.epilogue = atb::kMmGluBackward;
        dh.M = M; dh.N = F; dh.K = D; dh.act = act;
        dh.A[0] = {dY_dev, lddy}; dh.B[0] = {Wd_dev, ldwd};
        dh.G = G_dev; dh.U = U_dev; dh.keep32 = keep32;
        dh.C[0] = dG; dh.C[1] = dU; dh.ldc[0] = dh.ldc[1] = F;
        s = atb::mm_launch(&dh, 1, partial, st);
        if (s != ATB_OK) return s;
    }
    atb::MmProblem q[atb::kMmGroup];
    const int n = gradient_products(q, M, D, F, dX_dev, dWg_dev, dWd_dev);
    if (n == 0) return ATB_OK;
    atb::MmProblem* next = q;
    if (dX_dev) {
        atb::MmProblem& dx = *next++;
        dx.A[0] = {dG, F}; dx.A[1] = {dU, F}; dx.B[0] = {Wg_dev, ldw}; dx.B[1] = {Wu_dev, ldw};
        dx.C[0] = dX_dev; dx.ldc[0] = lddx;
    }
    if (dWg_dev) {
        atb::MmProblem& dw = *next++;
        dw.A[0] = {X_dev, ldx}; dw.B[0] = {dG, F}; dw.B[1] = {dU, F};
        dw.C[0] = dWg_dev; dw.C[1] = dWu_dev; dw.ldc[0] = dw.ldc[1] = lddw;
    }
    if (dWd_dev) {
        atb::MmProblem& dw = *next++;
        dw.A[0] = {H_dev, F}; dw.B[0] = {dY_dev, lddy};
        dw.C[0] = dWd_dev; dw.ldc[0] = lddwd;
    }
    return atb::mm_launch(q, n, partial, st);
}
