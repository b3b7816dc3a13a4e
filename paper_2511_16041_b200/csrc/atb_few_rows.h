// Internal interface of the few-row products (atb_few_rows.cu).  Not part of the ABI.
#pragma once
#include <cuda_runtime.h>

#include "atb_internal.h"

namespace atb {

constexpr int64_t kFewRows = 2;      // the most rows

// Y = X W (W [K][N]), and H = act(X Wg) * (X Wu) with the two products in G and U where those are not NULL (H, G, U [M][N]).
// weights_settled: the kernel ahead on the stream is one of this library's, which waits for all before it and does not write W;
// W is then fetched while that kernel still runs.
// M <= kFewRows; the alignment rules of the entry points (16 bytes, leading dimensions, K and N multiples of 8).
atb_status_t few_rows_product(int64_t M, int64_t K, int64_t N, const void* X, int64_t ldx, const void* W, int64_t ldw, void* Y, int64_t ldy,
                              bool weights_settled, cudaStream_t stream);
atb_status_t few_rows_glu(int64_t M, int64_t K, int64_t N, int act, const void* X, int64_t ldx, const void* Wg, const void* Wu, int64_t ldw, void* H,
                          void* G, void* U, cudaStream_t stream);

}  // namespace atb
