// Internal interface of the BF16 x BF16 product kernels (atb_bf16_mm_sm100.cu), used by the gated feed-forward block, the linear
// cross entropy and the linear layer.  Not part of the ABI.
#pragma once
#include <cuda_runtime.h>

#include "atb_internal.h"

namespace atb {

// A bf16 operand of C = A x B.  Stored as [M or N][K] rows (K runs along a row) or as [K][M or N] rows.
struct MmOperand {
    const void* base = nullptr;
    int64_t ld = 0;              // elements between rows
};

enum MmLayout {
    kMmNN = 0,                   // A[M][K], B[K][N]
    kMmNT = 1,                   // A[M][K], B[N][K]
    kMmTN = 2,                   // A[K][M], B[K][N]
};

enum MmEpilogue {
    kMmStore = 0,                // C (bf16)
    kMmAccumulate = 1,           // C32 (fp32), first: written, else added to
    kMmGlu = 2,                  // h = act(g) u from two products that share A; g and u too where wanted
    kMmGluBackward = 3,          // the product is dh; with the saved g and u: dg, du
    kMmRowStats = 4,             // per row and group of columns: maximum and sum of exp(c - maximum); the label's c
    kMmDlogits = 5,              // (exp(c - lse) - [column is the label]) * scale / unit (bf16)
    kMmLinear = 6,               // act(c + bias) + residual; c + bias too where wanted
};

struct MmProblem {
    MmLayout layout = kMmNN;
    MmEpilogue epilogue = kMmStore;
    int64_t M = 0, N = 0, K = 0;      // of one segment
    int k_segs = 1;                   // 2: C = A[0] x B[0] + A[1] x B[1]
    int n_segs = 1;                   // 2: C[0] = A[0] x B[0], C[1] = A[0] x B[1]  (kMmGlu always has two products)
    MmOperand A[2], B[2];
    void* C[3] = {nullptr, nullptr, nullptr};   // bf16 outputs; kMmGlu: h, g, u (g and u may be NULL, or FP32); kMmGluBackward: dg, du;
                                                // kMmLinear: the result, and the sum before the activation or NULL
    int64_t ldc[3] = {0, 0, 0};
    // kMmAccumulate
    float* C32 = nullptr;             // [M][N]
    bool first = true;                // kMmDlogits: finds *unit and writes it; else reads it
    const float* factor = nullptr;    // kMmStore, kMmAccumulate: the product is multiplied by *factor where given
    // kMmGlu, kMmGluBackward
    int act = 0;
    const void *G = nullptr, *U = nullptr;      // [M][N]
    bool keep32 = false;              // g and u in memory are FP32, else bf16
    // kMmLinear
    bool y32 = false, z32 = false, bias32 = false;      // result and residual, C[1], bias in FP32, else bf16
    const void* bias = nullptr;       // [N] or NULL
    const void* R = nullptr;          // [M][ldr] or NULL
    int64_t ldr = 0;
    // kMmRowStats, kMmDlogits: columns are the words col0 .. col0 + N - 1
    const int64_t* labels = nullptr;
    int64_t ignore_index = 0, col0 = 0;
    float2* stats = nullptr;          // [M][stats_ld]
    int64_t stats_ld = 0;
    float* label_logit = nullptr;     // [M]
    const float *lse = nullptr, *scale = nullptr;
    float* unit = nullptr;            // kMmDlogits: largest finite |scale| of the rows that count, 1 where that is 0
};

// The sizes alone, for the plans below.
inline MmProblem mm_sizes(MmLayout layout, MmEpilogue epilogue, int64_t M, int64_t N, int64_t K, int k_segs = 1, int n_segs = 1) {
    MmProblem q;
    q.layout = layout; q.epilogue = epilogue; q.M = M; q.N = N; q.K = K; q.k_segs = k_segs; q.n_segs = n_segs;
    return q;
}

constexpr int kMmGroup = 3;           // most products of one launch

// Entries of `stats` per row for a product of M x N x K.
int64_t mm_stats_per_row(int64_t M, int64_t N, int64_t K);
// Bytes of FP32 sums that a launch of these n products needs room for: 0 where none is split along K.
size_t mm_partial_bytes(const MmProblem* q, int n);

// Enqueues n <= kMmGroup products that do not depend on one another as one launch (and one more that joins the sums of
// those that are split along K): any number of kMmStore and kMmAccumulate products, or one of another kind.
// Pointers 16-byte aligned, leading dimensions multiples of 8 (callers check).  partial: mm_partial_bytes(q, n) bytes.
atb_status_t mm_launch(const MmProblem* q, int n, void* partial, cudaStream_t stream);

}  // namespace atb
