// Internal interface of the few-row products (atb_few_rows.cu).  Not part of the ABI.
#pragma once
#include <cuda_runtime.h>

#include "atb_internal.h"

namespace atb {

// The most rows.  Both products of a block, this form / the tensor cores (us, back to back on weights from memory):
//              512 x 1024    2048 x 5464    4096 x 10944    8192 x 24576
//   1 row      6.3 / 13.5    17.5 / 24.9    45.5 / 57.2      194 / 191
//   2 rows     7.0 / 13.5    19.0 / 25.0    47.7 / 58.0      208 / 199
//   3 rows     7.5 / 13.6    23.7 / 25.0    54.0 / 58.0      278 / 200
//   4 rows     8.7 / 13.6    34.4 / 25.0    79.6 / 58.2      412 / 207
// (3 and 4 rows in kernels built for the comparison: the rows' sums take the registers of the loads in flight.)  Two is what loses
// nowhere by more than a twentieth.
constexpr int64_t kFewRows = 2;

// Y = X W (W [K][N]), and H = act(X Wg) * (X Wu) with the two products in G and U where those are not NULL (H, G, U [M][N]; G and U
// FP32 with keep32, else bf16).
// weights_settled: the kernel ahead on the stream is one of this library's, which waits for all before it and does not write W;
// W is then fetched while that kernel still runs.
// M <= kFewRows; the alignment rules of the entry points (16 bytes, leading dimensions, K and N multiples of 8).
atb_status_t few_rows_product(int64_t M, int64_t K, int64_t N, const void* X, int64_t ldx, const void* W, int64_t ldw, void* Y, int64_t ldy,
                              bool weights_settled, cudaStream_t stream);
atb_status_t few_rows_glu(int64_t M, int64_t K, int64_t N, int act, const void* X, int64_t ldx, const void* Wg, const void* Wu, int64_t ldw, void* H,
                          void* G, void* U, bool keep32, cudaStream_t stream);

}  // namespace atb
