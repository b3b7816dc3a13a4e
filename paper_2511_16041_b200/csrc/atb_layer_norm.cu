// Layer norm, forward (values or BFP16 planes) and backward (sm_100a).
//
//   mu = sum(x) / N,  v = sum((x - mu)^2) / N,  r = 1 / sqrt(v + eps),  z = (x - mu) r,  y = z w + b
//   g = dy w,  dx = r (g - sum(g) / N - z sum(g z) / N),  dw = sum over rows of dy z,  db = sum over rows of dy
//
// Bound by memory: the forward pass reads x and writes y, the backward pass reads dy and x and writes dx, and
// nothing else of that size moves.  TPR threads share a row, at most kElems elements each, in registers: mean,
// variance and result take one read.  Blocks stay and walk rows blockIdx.x, + gridDim.x, ...: a thread keeps the same
// columns, so that w and b are loaded once and dw and db add up in registers, and the next rows (forward 3 of bf16, 2 of FP32; backward 3 and
// 2, but 2 of bf16 with 1024 threads and 1 of FP32 with 768) are on their way into shared memory (cp.async) while a row is worked on.  Rows on 16-byte boundaries: a thread copies what it will
// read itself, so that no barrier is needed.  Other rows are copied in 16-byte pieces all the same, from the boundary below
// their first element on, and read element by element from there.
// The variance is summed around means: of a warp's elements around their own mean in registers, and the warps' pairs
// (mean, sum of squares) joined by sum n_w (mean_w - mu)^2, in one exchange; sum(x^2) - N mu^2 would lose its digits
// where |mu| >> sqrt(v).  Means are quotients, not products with a rounded 1 / N, and z is made of distances to a mean, so that z is 0
// where all elements are one number (x r - mu r by one fma is off by the rounding of mu r: 1e-3 for rows of 100).  All sums are FP32.  Rows wider than the widest kernel are read again for every sum (*_wide kernels).
// Blocks write their sums of dw and db to the workspace, a second kernel adds those up in a fixed order: no atomics,
// the same bits on every call.
// Measured (compulsory bytes, of a measured copy rate of 6.55 TB/s): 16384 x 8192 bf16, FP32 weights: forward 96 us, 5.6 TB/s,
// backward 139 us, 5.8 TB/s; 8192 x 8192 FP32: 97 and 132 us, 5.5 and 6.1 TB/s; 8192 x 4096 bf16: 28 and 41 us, 4.8 TB/s;
// 12265 x 2499 off 16-byte boundaries: FP32 45 and 70 us, 5.4 and 5.2 TB/s, bf16 39 and 56 us, 3.1 and 3.3 TB/s (bound by
// instructions: an element at a time; groups of 8 shifted into place on both ways through shared memory took 48 and 73 us).  With one block per row and nothing on its way the first of these took 117 and 268 us.
// BFP16 planes: 8192 x 4096 from bf16 41 us, 2.6 TB/s, from FP32 47 us, 3.7 TB/s (bound by the block quantiser's instructions).  The *_wide
// kernels, 4096 x 20000: forward 93 us bf16 (3.5 TB/s), 173 us FP32; backward 343 us for both types, an element at a time.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "atb_internal.h"
#include "bfp16_block.cuh"
#include "dependent_launch.cuh"
#include "f32x2.cuh"

#include <type_traits>

namespace {

constexpr int kElems = 16;           // most elements of a row per thread
// Threads per row: the fewest that hold it, so that a thread has 11 to 16 elements.  8192 rows of 6000 bf16 elements take 37.7 us
// forward with 384 threads, 44.5 us with 512; 65536 rows of 1024 45 us with 64, 57 us with 128 threads of 8 elements.
constexpr int kThreadCounts[] = {32, 64, 96, 128, 192, 256, 384, 512, 768, 1024};
// Single elements of a thread that lie inside every row that `tpr` threads get: they need no test against N.  12265 x 2499 bf16 forward
// 39 instead of 43 us, 131072 x 333 55 instead of 72, 5000 x 12001 backward 128 instead of 164.  (32 threads also take rows
// of half their elements, in kernels of nv groups that hold no more.)  Groups of 8 need two tests in all, and without the
// first the compiler kept more alive than 64 registers hold: 16384 x 8192 101 instead of 93 us.
__host__ __device__ constexpr int full_groups(int tpr, int vec, int nv) {
    if (vec > 1) return 0;
    int fewer = tpr == 32 && nv * vec == kElems ? 16 : 0;
    for (const int t : kThreadCounts)
        if (t < tpr) fewer = t;
    const int full = fewer * kElems / tpr;
    return full < nv ? full : nv;
}
// Rows on their way per block: what the shared memory holds beside the row in hand.
template <class T, int TPR>
constexpr int kAhead = sizeof(T) == 2 ? (TPR < 1024 ? 3 : 2) : (TPR < 768 ? 2 : 1);
template <class T, int TPR>
constexpr int kAheadFwd = sizeof(T) == 2 ? 3 : 2;

// Blocks that stay on an SM: about 100 KB of rows on their way in each kernel.
// vec: rows on 16-byte boundaries; an element at a time takes 80 registers (forward) instead of 64.
__host__ __device__ constexpr int blocks_per_sm(int tpr, bool backward, bool vec) {
    switch (tpr) {
        case 32: return backward ? 3 : 6;              // four rows of 32 threads
        case 64: return backward ? 8 : 12;
        case 96: return backward ? 5 : vec ? 10 : 8;
        case 128: return backward ? 4 : vec ? 8 : 6;
        case 192: return backward ? 2 : vec ? 5 : 4;
        case 256: return backward ? 2 : vec ? 4 : 3;
        case 384: return backward ? 1 : 2;
        case 512: return backward || !vec ? 1 : 2;
        default: return 1;
    }
}

// ---------------------------------------------------------------------------------- loads and stores
// VEC consecutive elements as they are in memory: 8 (accesses of 16 bytes) or 1.
template <class T, int VEC>
struct Raw {
    uint32_t w[VEC * sizeof(T) / 4];
};
template <>
struct Raw<__nv_bfloat16, 1> {
    uint16_t w[1];
};

template <class T, int VEC>
__device__ __forceinline__ void load_raw(const T* p, Raw<T, VEC>& r) {
    constexpr int BYTES = static_cast<int>(sizeof(T)) * VEC;
    if constexpr (BYTES >= 16) {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const uint4 u = reinterpret_cast<const uint4*>(p)[i];
            r.w[4 * i] = u.x; r.w[4 * i + 1] = u.y; r.w[4 * i + 2] = u.z; r.w[4 * i + 3] = u.w;
        }
    } else if constexpr (BYTES == 4) {
        r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        r.w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
}
template <class T, int VEC>
__device__ __forceinline__ void to_float(const Raw<T, VEC>& r, float (&v)[VEC]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = __uint_as_float(r.w[i]);
    } else if constexpr (VEC > 1) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            v[2 * i] = __uint_as_float(r.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
        }
    } else {
        v[0] = __uint_as_float(static_cast<uint32_t>(r.w[0]) << 16);
    }
}
template <class T, int VEC>
__device__ __forceinline__ void load_f(const T* p, float (&v)[VEC]) {
    Raw<T, VEC> r;
    load_raw(p, r);
    to_float(r, v);
}
// Columns n .. n + VEC - 1 of a vector of N weights, or `none` where there is no vector.
template <class T, int VEC>
__device__ __forceinline__ void load_or(const T* p, int64_t n, int64_t N, float none, Raw<T, VEC>& r) {
    const uint32_t bits = __float_as_uint(none), half = bits >> 16;
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(r.w) / sizeof(r.w[0])); ++i) {
        if constexpr (sizeof(T) == 4) r.w[i] = bits;
        else if constexpr (VEC == 1) r.w[i] = static_cast<uint16_t>(half);
        else r.w[i] = half | half << 16;
    }
    if (p && n < N) load_raw<T, VEC>(p + n, r);
}
// What a thread keeps of them: as they are in memory, or, one by one, in FP32 (a register each either way).
template <class T, int VEC>
using Kept = std::conditional_t<VEC == 1, float, T>;
template <class T, int VEC>
__device__ __forceinline__ void keep_or(const T* p, int64_t n, int64_t N, float none, Raw<Kept<T, VEC>, VEC>& r) {
    if constexpr (VEC == 1 && sizeof(T) == 2) {
        Raw<T, 1> raw;
        load_or<T, 1>(p, n, N, none, raw);
        // kept: the compiler otherwise widens them again in every row
        asm volatile("shl.b32 %0, %1, 16;" : "=r"(r.w[0]) : "r"(static_cast<uint32_t>(raw.w[0])));
    } else {
        load_or<T, VEC>(p, n, N, none, r);
    }
}
template <class T, int VEC>
__device__ __forceinline__ void store_f(T* p, const float (&v)[VEC]) {
    if constexpr (sizeof(T) == 4) {
        if constexpr (VEC > 1) {
#pragma unroll
            for (int i = 0; i < VEC / 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
            *p = v[0];
        }
    } else if constexpr (VEC > 1) {
        uint32_t o[VEC / 2];
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const __nv_bfloat162 b2 = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            o[i] = *reinterpret_cast<const uint32_t*>(&b2);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
    } else {
        *p = __float2bfloat16_rn(v[0]);
    }
}

// ---------------------------------------------------------------------------------- pairs
// The backward kernel works on its elements in pairs by the two-wide FP32 instructions, which round each half like the scalar
// ones: 3 to 10 % faster than scalar arithmetic.  (The forward kernel, with half the arithmetic per byte, was 5 to 15 %
// slower in this form.)
using namespace f32x2;

// A thread's elements as pairs: NV groups of VEC, pairs of neighbours (VEC = 8) or of one element each of two groups (VEC = 1).
template <class T, int VEC, int NV>
__device__ __forceinline__ void to_pairs(const Raw<T, VEC> (&r)[NV], float2 (&v)[NV * VEC / 2]) {
    static_assert(NV * VEC % 2 == 0, "");
    if constexpr (VEC == 1) {
#pragma unroll
        for (int i = 0; i < NV; i += 2) {
            float a[1], b[1];
            to_float(r[i], a);
            to_float(r[i + 1], b);
            v[i / 2] = make_float2(a[0], b[0]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float f[VEC];
            to_float(r[i], f);
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e) v[i * VEC / 2 + e] = make_float2(f[2 * e], f[2 * e + 1]);
        }
    }
}
// Group i of them.
template <int VEC, int P>
__device__ __forceinline__ void group(const float2 (&v)[P], int i, float (&f)[VEC]) {
    if constexpr (VEC == 1) {
        f[0] = i & 1 ? v[i / 2].y : v[i / 2].x;
    } else {
#pragma unroll
        for (int e = 0; e < VEC / 2; ++e) { f[2 * e] = v[i * VEC / 2 + e].x; f[2 * e + 1] = v[i * VEC / 2 + e].y; }
    }
}
template <class T, int VEC>
__device__ __forceinline__ void clear(Raw<T, VEC>& r) {
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(r.w) / sizeof(r.w[0])); ++i) r.w[i] = 0;
}

// ---------------------------------------------------------------------------------- sums over a row's threads
template <int K>
__device__ __forceinline__ void warp_sum(float (&v)[K]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
}
// s / n from inv = 1 / n: the product's remainder, which an fma gives exactly, takes it to the quotient where that is a number of
// FP32 (and to the nearest but for rare ties of its rounding), without a division's branches.  An infinite sum stays what it is.
__device__ __forceinline__ float quotient(float s, float n, float inv) {
    const float q = s * inv;
    return fabsf(q) <= 3.402823466e38f ? fmaf(fmaf(-q, n, s), inv, q) : q;
}
// Every thread of the row gets the sum of K values over the TPR threads.  TPR = 32: one warp; else the whole block,
// through `red`, of which a row takes another slice than the row before it (a slice is written again only after a
// barrier that follows its last read).
template <int TPR, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float (*red)[K]) {
    warp_sum(v);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) red[warp][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = lane < W ? red[lane][k] : 0.f;
#pragma unroll
            for (int o = W > 16 ? 16 : W > 8 ? 8 : W > 4 ? 4 : W > 2 ? 2 : 1; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
            v[k] = __shfl_sync(0xFFFFFFFFu, v[k], 0);
        }
    }
}

// ---------------------------------------------------------------------------------- rows on their way
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// VEC = 8: NV groups of 8 elements per thread and row, group i of thread t at column (i TPR + t) 8.  A bf16 group is one
// 16-byte piece, which the thread copies itself; the 64 pieces of a warp's FP32 groups are copied by the warp, 512
// consecutive bytes at a time.
template <class T, int VEC, int TPR, int NV>
struct RowSource {
    static_assert(VEC == 8, "");
    static constexpr int CHUNKS = static_cast<int>(sizeof(T)) / 2;
    static constexpr bool SHARED = CHUNKS == 2;        // a thread reads what others of its warp have copied
    static constexpr int THREADS = TPR == 32 ? 128 : TPR;
    static constexpr uint32_t STAGE_BYTES = THREADS * NV * CHUNKS * 16;
    uint32_t base;                                     // this warp's first slot
    const T* first;
    int64_t ld;
    int N, col;                                        // col: first column of this lane's first piece
    __device__ __forceinline__ RowSource(uint32_t smem, const void* x, int64_t ld_, int64_t, int N_, int t)
        : base(smem + (threadIdx.x & ~31u) * CHUNKS * 16), first(static_cast<const T*>(x)), ld(ld_), N(N_),
          col((t & ~31) * 8 + (t & 31) * (8 / CHUNKS)) {}
    __device__ __forceinline__ void fetch(int stage, int64_t m) const {
        const T* row = first + m * ld + col;
        const uint32_t dst = base + stage * STAGE_BYTES + (threadIdx.x & 31) * 16;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
                if (col + i * TPR * 8 + c * 128 < N) copy16(dst + i * CHUNKS * THREADS * 16 + c * 512, row + i * TPR * 8 + c * 128);
    }
    __device__ __forceinline__ void read(int stage, int64_t, int i, Raw<T, VEC>& r) const {
        const uint32_t at = base + stage * STAGE_BYTES + i * CHUNKS * THREADS * 16 + (threadIdx.x & 31) * CHUNKS * 16;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[4 * c]), "=r"(r.w[4 * c + 1]), "=r"(r.w[4 * c + 2]), "=r"(r.w[4 * c + 3])
                         : "r"(at + 16 * c) : "memory");
    }
};
// VEC = 1: element i TPR + t of the row, wherever the row starts.  The row's threads copy the 16-byte pieces that cover it; what
// a piece holds besides the row is not read, and a row with a piece that is not wholly inside the matrix is copied by elements.
template <class T, int TPR, int NV>
struct RowSource<T, 1, TPR, NV> {
    static constexpr bool SHARED = true;
    static constexpr uint32_t ROW_BYTES = TPR * NV * sizeof(T) + 16, STAGE_BYTES = (TPR == 32 ? 4 : 1) * ROW_BYTES;
    uint32_t base;
    const T* first;
    int64_t ld;
    uintptr_t end;                                     // of the matrix
    int N, t;
    __device__ __forceinline__ RowSource(uint32_t smem, const void* x, int64_t ld_, int64_t M, int N_, int t_)
        : base(smem + (TPR == 32 ? threadIdx.x >> 5 : 0) * ROW_BYTES), first(static_cast<const T*>(x)), ld(ld_),
          end(reinterpret_cast<uintptr_t>(first + (M - 1) * ld + N_)), N(N_), t(t_) {}
    __device__ __forceinline__ void fetch(int stage, int64_t m) const {
        const uintptr_t row = reinterpret_cast<uintptr_t>(first + m * ld), from = row & ~static_cast<uintptr_t>(15);
        const uint32_t skip = static_cast<uint32_t>(row - from);
        const int bytes = static_cast<int>(skip + N * sizeof(T));                   // from `from` to the row's end
        const uint32_t dst = base + stage * STAGE_BYTES;
        if (from >= reinterpret_cast<uintptr_t>(first) && from + ((bytes + 15) & ~15) <= end) {
            constexpr int ROUNDS = static_cast<int>((NV * sizeof(T) + 15) / 16 + 1);      // of TPR pieces, most
#pragma unroll
            for (int k = 0; k < ROUNDS; ++k) {
                const int o = 16 * (t + k * TPR);
                if (o < bytes) copy16(dst + o, reinterpret_cast<const char*>(from) + o);
            }
        } else {
            for (int n = t; n < N; n += TPR) {
                const uint32_t to = dst + skip + n * static_cast<uint32_t>(sizeof(T));
                if constexpr (sizeof(T) == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(reinterpret_cast<const uint32_t*>(row)[n]) : "memory");
                else asm volatile("st.shared.b16 [%0], %1;" ::"r"(to), "h"(reinterpret_cast<const uint16_t*>(row)[n]) : "memory");
            }
        }
    }
    __device__ __forceinline__ void read(int stage, int64_t m, int i, Raw<T, 1>& r) const {
        const uint32_t at = base + stage * STAGE_BYTES + (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(first + m * ld)) & 15u) + t * static_cast<uint32_t>(sizeof(T));
        if constexpr (sizeof(T) == 4) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r.w[0]) : "r"(at + i * TPR * 4) : "memory");
        else asm volatile("ld.shared.b16 %0, [%1];" : "=h"(r.w[0]) : "r"(at + i * TPR * 2) : "memory");
    }
};
// Between this thread's wait for its copies and its reads: the other threads' copies have landed too.  Between reads that no sum over
// the row's threads follows and the next copies into their stage: the other threads have read.
template <class Source, int VEC, int TPR>
__device__ __forceinline__ void row_barrier() {
    if constexpr (Source::SHARED) {
        if constexpr (VEC == 1 && TPR > 32) __syncthreads(); else __syncwarp();
    }
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// ---------------------------------------------------------------------------------- forward
struct FwdParams {
    int64_t M, N, ldx, ldy, rows;          // rows: rows the grid covers (M, or M padded for the BFP16 planes)
    const void *x, *w, *b;
    float eps;
    void* y;                               // values, or the mantissa plane
    uint8_t* exp;                          // BFP16: exponent plane
    float *mean, *rstd;
};

// One BFP16 block of row m, columns n .. n + 7.
__device__ __forceinline__ void put_block(const FwdParams& p, int64_t m, int64_t n, const float (&v)[8]) {
    uint32_t packed[2];
    const int E = bfp16::quantize_block8(v, packed);
    *reinterpret_cast<uint2*>(static_cast<int8_t*>(p.y) + m * p.N + n) = make_uint2(packed[0], packed[1]);
    p.exp[((n >> 6) * p.rows + m) * 8 + ((n >> 3) & 7)] = static_cast<uint8_t>(E);
}
// The exponent plane's padding of row m: blocks past the last column, and whole rows past M.
__device__ __forceinline__ void put_exp_padding(const FwdParams& p, int64_t m, int t, int threads) {
    const int64_t first = m < p.M ? p.N >> 3 : 0, last = ((p.N + 63) >> 6) * 8;
    for (int64_t j = first + t; j < last; j += threads) p.exp[((j >> 3) * p.rows + m) * 8 + (j & 7)] = 0;
}
template <class TX, class TW, int VEC, int TPR, int NV, bool BFP>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, blocks_per_sm(TPR, false, VEC > 1)) layer_norm_kernel(const FwdParams p) {
    using Source = RowSource<TX, VEC, TPR, NV>;
    constexpr int WALKERS = TPR == 32 ? 4 : 1, W = TPR / 32;
    constexpr int STAGES = kAheadFwd<TX, TPR> + 1, FULL = full_groups(TPR, VEC, NV);
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float2 red[2][W];
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x, lane = threadIdx.x & 31, warp = TPR == 32 ? 0 : threadIdx.x >> 5;
    const int N = static_cast<int>(p.N), col = t * VEC;                 // group i: columns col + i TPR VEC ..
    const int64_t first = static_cast<int64_t>(blockIdx.x) * WALKERS + (TPR == 32 ? threadIdx.x >> 5 : 0), step = static_cast<int64_t>(gridDim.x) * WALKERS;
    const Source src(sm100::smem_u32(ring), p.x, p.ldx, p.M, N, t);
    // elements of warp `lane` (join) and of this warp (the mean that its squares are summed around)
    int count = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) count += max(0, min(32 * VEC, N - (i * TPR + lane * 32) * VEC));
    if (lane >= W) count = 0;
    const float elems = static_cast<float>(count), inv_n = 1.f / static_cast<float>(N);
    const int own = __shfl_sync(0xFFFFFFFFu, count, warp);
    const float inv_own = own > 0 ? 1.f / static_cast<float>(own) : 0.f;
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
#pragma unroll
    for (int s = 0; s < kAheadFwd<TX, TPR>; ++s) {
        if (first + s * step < p.M) src.fetch(s, first + s * step);
        async_commit();
    }
    Raw<Kept<TW, VEC>, VEC> w[NV], b[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        keep_or<TW, VEC>(static_cast<const TW*>(p.w), col + i * TPR * VEC, N, 1.f, w[i]);
        keep_or<TW, VEC>(static_cast<const TW*>(p.b), col + i * TPR * VEC, N, 0.f, b[i]);
    }
    int stage = 0, turn = 0;
    for (int64_t m = first; m < p.rows; m += step, turn ^= 1) {
        if constexpr (BFP) put_exp_padding(p, m, t, TPR);
        if (m < p.M) {                     // the same for all threads of the row
            const int ahead = stage == 0 ? kAheadFwd<TX, TPR> : stage - 1;       // the stage that the row before this one has left
            if (m + kAheadFwd<TX, TPR> * step < p.M) src.fetch(ahead, m + kAheadFwd<TX, TPR> * step);
            async_commit();
            async_wait<kAheadFwd<TX, TPR>>();
            row_barrier<Source, VEC, TPR>();
            float v[NV][VEC], s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i < FULL || col + i * TPR * VEC < N) {
                    Raw<TX, VEC> raw;
                    src.read(stage, m, i, raw);
                    to_float(raw, v[i]);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) s[0] += v[i][e];
                }
            }
            warp_sum(s);
            const float mine = quotient(s[0], __shfl_sync(0xFFFFFFFFu, elems, warp), inv_own);       // the mean of the warp's elements
            s[0] = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (i < FULL || col + i * TPR * VEC < N)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        v[i][e] -= mine;
                        s[0] += v[i][e] * v[i][e];
                    }
            warp_sum(s);
            float mu = mine;
            if constexpr (TPR > 32) {
                if (lane == 0) red[turn][warp] = make_float2(mine, s[0]);
                __syncthreads();
                // every warp joins the warps' pairs: lane l has warp l's
                const float2 part = lane < W ? red[turn][lane] : make_float2(0.f, 0.f);
                float sum[1] = {elems * part.x};
                warp_sum(sum);
                mu = quotient(sum[0], static_cast<float>(N), inv_n);
                s[0] = part.y + elems * (part.x - mu) * (part.x - mu);
                warp_sum(s);
            }
            const float r = rsqrtf(s[0] * inv_n + p.eps);
            if (t == 0) {
                if (p.mean) p.mean[m] = mu;
                if (p.rstd) p.rstd[m] = r;
            }
            // z = (x - mu) r from the distances to the warp's mean
            const float shift = (mine - mu) * r;
            TX* const y = BFP ? nullptr : static_cast<TX*>(p.y) + m * p.ldy + col;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i < FULL || col + i * TPR * VEC < N) {
                    float fw[VEC], fb[VEC];
                    to_float<Kept<TW, VEC>, VEC>(w[i], fw);
                    to_float<Kept<TW, VEC>, VEC>(b[i], fb);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v[i][e] = fmaf(fmaf(v[i][e], r, shift), fw[e], fb[e]);
                    if constexpr (BFP) put_block(p, m, col + i * TPR * VEC, v[i]);
                    else store_f<TX, VEC>(y + i * TPR * VEC, v[i]);
                }
            }
            stage = stage + 1 == STAGES ? 0 : stage + 1;
        }
    }
}

// Any width: the row is read once for each of mean, variance and result.
template <class TX, class TW, int VEC, bool BFP>
__global__ void __launch_bounds__(1024) layer_norm_wide_kernel(const FwdParams p) {
    __shared__ float red[2][32][1];
    const int64_t m = blockIdx.x;
    if constexpr (BFP) {
        put_exp_padding(p, m, threadIdx.x, 1024);
        if (m >= p.M) return;
    }
    const TX* x = static_cast<const TX*>(p.x) + m * p.ldx;
    float s[1] = {0.f}, v[VEC];
    for (int64_t n = threadIdx.x * VEC; n < p.N; n += 1024 * VEC) {
        load_f<TX, VEC>(x + n, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[0] += v[e];
    }
    const float inv_n = 1.f / static_cast<float>(p.N);
    row_sum<1024, 1>(s, red[0]);
    const float mu = quotient(s[0], static_cast<float>(p.N), inv_n);
    s[0] = 0.f;
    for (int64_t n = threadIdx.x * VEC; n < p.N; n += 1024 * VEC) {
        load_f<TX, VEC>(x + n, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[0] += (v[e] - mu) * (v[e] - mu);
    }
    row_sum<1024, 1>(s, red[1]);
    const float r = rsqrtf(s[0] * inv_n + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[m] = mu;
        if (p.rstd) p.rstd[m] = r;
    }
    for (int64_t n = threadIdx.x * VEC; n < p.N; n += 1024 * VEC) {
        load_f<TX, VEC>(x + n, v);
        Raw<TW, VEC> raw;
        float fw[VEC], fb[VEC];
        load_or<TW, VEC>(static_cast<const TW*>(p.w), n, p.N, 1.f, raw);
        to_float(raw, fw);
        load_or<TW, VEC>(static_cast<const TW*>(p.b), n, p.N, 0.f, raw);
        to_float(raw, fb);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = fmaf((v[e] - mu) * r, fw[e], fb[e]);
        if constexpr (BFP) put_block(p, m, n, v);
        else store_f<TX, VEC>(static_cast<TX*>(p.y) + m * p.ldy + n, v);
    }
}

// ---------------------------------------------------------------------------------- backward
struct BwdParams {
    int64_t M, N, lddy, ldx, lddx;
    const void *dy, *x, *w;
    const float *mean, *rstd;
    void* dx;
    float* part;                           // [blocks][2][N]: sums of dw and db of each block
};

template <class TX, class TW, int VEC, int TPR, int NV>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, blocks_per_sm(TPR, true, VEC > 1)) layer_norm_backward_kernel(const BwdParams p) {
    using Source = RowSource<TX, VEC, TPR, NV>;
    constexpr int WALKERS = TPR == 32 ? 4 : 1, W = TPR / 32;
    constexpr int STAGES = kAhead<TX, TPR> + 1, P = NV * VEC / 2, FULL = full_groups(TPR, VEC, NV);
    // 768 and 1024 threads have 80 and 64 registers each: the row is read from shared memory again after the sums
    constexpr bool REREAD = TPR >= 768;
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float red[2][W][2];
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
    const int N = static_cast<int>(p.N), col = t * VEC;                 // group i: columns col + i TPR VEC ..
    const int64_t first = static_cast<int64_t>(blockIdx.x) * WALKERS + (TPR == 32 ? threadIdx.x >> 5 : 0), step = static_cast<int64_t>(gridDim.x) * WALKERS;
    const Source sx(sm100::smem_u32(ring), p.x, p.ldx, p.M, N, t), sd(sm100::smem_u32(ring) + STAGES * Source::STAGE_BYTES, p.dy, p.lddy, p.M, N, t);
    const float inv_n = 1.f / static_cast<float>(N);
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
#pragma unroll
    for (int s = 0; s < kAhead<TX, TPR>; ++s) {
        if (first + s * step < p.M) {
            sx.fetch(s, first + s * step);
            sd.fetch(s, first + s * step);
        }
        async_commit();
    }
    Raw<Kept<TW, VEC>, VEC> w[NV];
    float2 dw[P], db[P];
#pragma unroll
    for (int i = 0; i < NV; ++i) keep_or<TW, VEC>(static_cast<const TW*>(p.w), col + i * TPR * VEC, N, 1.f, w[i]);
#pragma unroll
    for (int k = 0; k < P; ++k) dw[k] = db[k] = make_float2(0.f, 0.f);
    int stage = 0, turn = 0;
    float mu = 0.f, r = 0.f;
    if (first < p.M) { mu = p.mean[first]; r = p.rstd[first]; }
    for (int64_t m = first; m < p.M; m += step, turn ^= 1) {
        const int ahead = stage == 0 ? kAhead<TX, TPR> : stage - 1;           // the stage that the row before this one has left
        if (m + kAhead<TX, TPR> * step < p.M) {
            sx.fetch(ahead, m + kAhead<TX, TPR> * step);
            sd.fetch(ahead, m + kAhead<TX, TPR> * step);
        }
        async_commit();
        float next_mu = 0.f, next_r = 0.f;
        if (m + step < p.M) { next_mu = p.mean[m + step]; next_r = p.rstd[m + step]; }
        async_wait<kAhead<TX, TPR>>();
        row_barrier<Source, VEC, TPR>();
        // z, dy and g = dy w of this thread; elements past the row's end have dy = 0 and count in no sum
        float2 z[P], g[P], s0 = make_float2(0.f, 0.f), s1 = s0;        // z: x - mu as loaded
        const float2 scale = both(r), shift = both(-mu);
        const auto load = [&] {
            Raw<TX, VEC> raw[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i < FULL || col + i * TPR * VEC < N) sx.read(stage, m, i, raw[i]);
                else clear(raw[i]);
            }
            to_pairs<TX, VEC, NV>(raw, z);
#pragma unroll
            for (int k = 0; k < P; ++k) z[k] = add2(z[k], shift);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i < FULL || col + i * TPR * VEC < N) sd.read(stage, m, i, raw[i]);
                else clear(raw[i]);
            }
            to_pairs<TX, VEC, NV>(raw, g);
        };
        load();
        {
            float2 f[P];
            to_pairs<Kept<TW, VEC>, VEC, NV>(w, f);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                z[k] = mul2(z[k], scale);
                dw[k] = fma2(g[k], z[k], dw[k]);
                db[k] = add2(db[k], g[k]);
                g[k] = mul2(g[k], f[k]);
                s0 = add2(s0, g[k]);
                s1 = fma2(g[k], z[k], s1);
            }
        }
        float s[2] = {s0.x + s0.y, s1.x + s1.y};
        row_sum<TPR, 2>(s, red[turn]);
        if (p.dx) {
            TX* const dx = static_cast<TX*>(p.dx) + m * p.lddx + col;
            const float m0 = s[0] * inv_n, m1 = s[1] * inv_n;
            if constexpr (REREAD) {        // r (dy w - m0 - (x - mu) (r m1))
                load();
                float2 f[P];
                to_pairs<Kept<TW, VEC>, VEC, NV>(w, f);
                const float2 c0 = both(-m0), c1 = both(-r * m1);
#pragma unroll
                for (int k = 0; k < P; ++k) g[k] = mul2(fma2(z[k], c1, fma2(g[k], f[k], c0)), scale);
            } else {                       // r g - r m0 - z (r m1)
                const float2 c0 = both(-r * m0), c1 = both(-r * m1);
#pragma unroll
                for (int k = 0; k < P; ++k) g[k] = fma2(z[k], c1, fma2(g[k], scale, c0));
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (i < FULL || col + i * TPR * VEC < N) {
                    float f[VEC];
                    group<VEC, P>(g, i, f);
                    store_f<TX, VEC>(dx + i * TPR * VEC, f);
                }
            }
        }
        // the row's stage is the next to be filled, by other threads than those that have just read it again
        if constexpr (REREAD) row_barrier<Source, VEC, TPR>();
        mu = next_mu;
        r = next_r;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    if (p.part) {                          // a walker's sums: [walker][2][N]
        float* out = p.part + first * 2 * p.N + col;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i < FULL || col + i * TPR * VEC < N) {
                float f[VEC];
                group<VEC, P>(dw, i, f);
                store_f<float, VEC>(out + i * TPR * VEC, f);
                group<VEC, P>(db, i, f);
                store_f<float, VEC>(out + p.N + i * TPR * VEC, f);                 // N is a multiple of VEC
            }
        }
    }
}

// Any width, dx: a block per row, which is read for the sums and again for the result.
template <class TX, class TW>
__global__ void __launch_bounds__(1024) layer_norm_backward_wide_kernel(const BwdParams p) {
    __shared__ float red[32][2];
    const int64_t m = blockIdx.x;
    const TX* x = static_cast<const TX*>(p.x) + m * p.ldx;
    const TX* dy = static_cast<const TX*>(p.dy) + m * p.lddy;
    TX* dx = static_cast<TX*>(p.dx) + m * p.lddx;
    const float mu = p.mean[m], r = p.rstd[m], inv_n = 1.f / static_cast<float>(p.N);
    float s[2] = {0.f, 0.f}, vx[1], vd[1], w[1] = {1.f};
    for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
        load_f<TX, 1>(x + n, vx);
        load_f<TX, 1>(dy + n, vd);
        if (p.w) load_f<TW, 1>(static_cast<const TW*>(p.w) + n, w);
        s[0] += vd[0] * w[0];
        s[1] += vd[0] * w[0] * ((vx[0] - mu) * r);
    }
    row_sum<1024, 2>(s, red);
    for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
        load_f<TX, 1>(x + n, vx);
        load_f<TX, 1>(dy + n, vd);
        if (p.w) load_f<TW, 1>(static_cast<const TW*>(p.w) + n, w);
        vx[0] = r * (vd[0] * w[0] - s[0] * inv_n - (vx[0] - mu) * r * (s[1] * inv_n));
        store_f<TX, 1>(dx + n, vx);
    }
}
// Any width, dw and db: a block takes 256 columns and every gridDim.y-th row.
template <class TX>
__global__ void __launch_bounds__(256) layer_norm_backward_columns_kernel(const BwdParams p) {
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (n >= p.N) return;
    float dw = 0.f, db = 0.f, vx[1], vd[1];
    for (int64_t m = blockIdx.y; m < p.M; m += gridDim.y) {
        load_f<TX, 1>(static_cast<const TX*>(p.x) + m * p.ldx + n, vx);
        load_f<TX, 1>(static_cast<const TX*>(p.dy) + m * p.lddy + n, vd);
        dw += vd[0] * ((vx[0] - p.mean[m]) * p.rstd[m]);
        db += vd[0];
    }
    float* out = p.part + static_cast<int64_t>(blockIdx.y) * 2 * p.N;
    out[n] = dw;
    out[p.N + n] = db;
}

// dw[n], db[n] = sum over the `parts` partial sums, in a fixed order: 32 columns of [dw | db] per block, 16 warps that
// take every 16th partial sum, then the 16 in turn.
constexpr int kSumWarps = 16;
template <class TW>
__global__ void __launch_bounds__(32 * kSumWarps) layer_norm_backward_sum_kernel(const float* part, int parts, int64_t N, TW* dw, TW* db) {
    __shared__ float s[kSumWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 32 + lane;
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
    float v = 0.f;
    if (c < 2 * N) {
#pragma unroll 8
        for (int i = warp; i < parts; i += kSumWarps) v += part[static_cast<int64_t>(i) * 2 * N + c];
    }
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < 2 * N) {
#pragma unroll
        for (int i = 1; i < kSumWarps; ++i) v += s[i][lane];
        TW* out = c < N ? dw : db;
        const float r[1] = {v};
        if (out) store_f<TW, 1>(out + (c < N ? c : c - N), r);
    }
}

// ---------------------------------------------------------------------------------- host
// Threads per row, at most `most`; 0: a wide kernel.
int threads_per_row(int64_t N, int most) {
    for (const int t : kThreadCounts)
        if (t <= most && N <= static_cast<int64_t>(t) * kElems) return t;
    return 0;
}
constexpr int kMostThreads = 1024;
// Backward, FP32: two rows of 16384 do not leave room for the next ones.
template <class TX>
constexpr int kBwdThreads = sizeof(TX) == 2 ? 1024 : 768;

// A kernel whose rows on their way may take more, with its static arrays, than the 48 KB of shared memory that need no leave.
template <class... Args>
cudaError_t launch_ring(void (*kernel)(Args...), unsigned grid, unsigned block, size_t smem, cudaStream_t stream, Args... args) {
    if (smem > 40 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return e;
    }
    return atb::launch_dependent(kernel, grid, block, 1u, smem, stream, args...);
}

template <class TX, class TW, int VEC, bool BFP, int TPR>
cudaError_t launch_fwd_rows(const FwdParams& p, cudaStream_t st) {
    constexpr int NV = kElems / VEC, HALF = NV / 2, THREADS = TPR == 32 ? 128 : TPR;
    const int64_t walkers = TPR == 32 ? 4 : 1, all = (p.rows + walkers - 1) / walkers, most = static_cast<int64_t>(atb::kSmCount) * blocks_per_sm(TPR, false, VEC > 1);
    const unsigned blocks = static_cast<unsigned>(all < most ? all : most);
    if constexpr (TPR == 32)               // the narrowest rows
        if (p.N <= TPR * kElems / 2)
            return launch_ring(layer_norm_kernel<TX, TW, VEC, TPR, HALF, BFP>, blocks, THREADS, (kAheadFwd<TX, TPR> + 1) * RowSource<TX, VEC, TPR, HALF>::STAGE_BYTES, st, p);
    return launch_ring(layer_norm_kernel<TX, TW, VEC, TPR, NV, BFP>, blocks, THREADS, (kAheadFwd<TX, TPR> + 1) * RowSource<TX, VEC, TPR, NV>::STAGE_BYTES, st, p);
}
template <class TX, class TW, int VEC, bool BFP>
cudaError_t launch_fwd(const FwdParams& p, cudaStream_t st) {
    switch (threads_per_row(p.N, kMostThreads)) {
        case 32: return launch_fwd_rows<TX, TW, VEC, BFP, 32>(p, st);
        case 64: return launch_fwd_rows<TX, TW, VEC, BFP, 64>(p, st);
        case 96: return launch_fwd_rows<TX, TW, VEC, BFP, 96>(p, st);
        case 128: return launch_fwd_rows<TX, TW, VEC, BFP, 128>(p, st);
        case 192: return launch_fwd_rows<TX, TW, VEC, BFP, 192>(p, st);
        case 256: return launch_fwd_rows<TX, TW, VEC, BFP, 256>(p, st);
        case 384: return launch_fwd_rows<TX, TW, VEC, BFP, 384>(p, st);
        case 512: return launch_fwd_rows<TX, TW, VEC, BFP, 512>(p, st);
        case 768: return launch_fwd_rows<TX, TW, VEC, BFP, 768>(p, st);
        case 1024: return launch_fwd_rows<TX, TW, VEC, BFP, 1024>(p, st);
    }
    layer_norm_wide_kernel<TX, TW, VEC, BFP><<<static_cast<unsigned>(p.rows), 1024, 0, st>>>(p);
    return cudaGetLastError();
}

// Blocks that walk the rows: one per SM and more while each walker still has 16 rows, since its sums of 8 N bytes go
// through the workspace.  The same on every host: the workspace's size depends on it.
int walking_blocks(int64_t M, int64_t N) {
    const int tpr = threads_per_row(N, kMostThreads);
    const int64_t walkers = tpr == 32 ? 4 : 1, all = (M + walkers - 1) / walkers, most = static_cast<int64_t>(atb::kSmCount) * blocks_per_sm(tpr, true, true);
    int64_t blocks = (M + 16 * walkers - 1) / (16 * walkers);
    if (blocks < atb::kSmCount) blocks = atb::kSmCount;
    if (blocks > most) blocks = most;
    if (blocks > all) blocks = all;
    return static_cast<int>(blocks < 1 ? 1 : blocks);
}
int partial_sums(int64_t M, int64_t N) {
    return walking_blocks(M, N) * (threads_per_row(N, kMostThreads) == 32 ? 4 : 1);
}

template <class TX, class TW, int VEC, int TPR>
cudaError_t launch_bwd_rows(const BwdParams& p, cudaStream_t st) {
    constexpr int NV = kElems / VEC, HALF = NV / 2, THREADS = TPR == 32 ? 128 : TPR;
    const unsigned blocks = static_cast<unsigned>(walking_blocks(p.M, p.N));
    if constexpr (TPR == 32)               // the narrowest rows
        if (p.N <= TPR * kElems / 2)
            return launch_ring(layer_norm_backward_kernel<TX, TW, VEC, TPR, HALF>, blocks, THREADS,
                           2 * (kAhead<TX, TPR> + 1) * RowSource<TX, VEC, TPR, HALF>::STAGE_BYTES, st, p);
    return launch_ring(layer_norm_backward_kernel<TX, TW, VEC, TPR, NV>, blocks, THREADS, 2 * (kAhead<TX, TPR> + 1) * RowSource<TX, VEC, TPR, NV>::STAGE_BYTES, st, p);
}
template <class TX, class TW, int VEC>
cudaError_t launch_bwd(const BwdParams& p, cudaStream_t st) {
    switch (threads_per_row(p.N, kBwdThreads<TX>)) {
        case 32: return launch_bwd_rows<TX, TW, VEC, 32>(p, st);
        case 64: return launch_bwd_rows<TX, TW, VEC, 64>(p, st);
        case 96: return launch_bwd_rows<TX, TW, VEC, 96>(p, st);
        case 128: return launch_bwd_rows<TX, TW, VEC, 128>(p, st);
        case 192: return launch_bwd_rows<TX, TW, VEC, 192>(p, st);
        case 256: return launch_bwd_rows<TX, TW, VEC, 256>(p, st);
        case 384: return launch_bwd_rows<TX, TW, VEC, 384>(p, st);
        case 512: return launch_bwd_rows<TX, TW, VEC, 512>(p, st);
        case 768: return launch_bwd_rows<TX, TW, VEC, 768>(p, st);
        case 1024:
            if constexpr (kBwdThreads<TX> == 1024) return launch_bwd_rows<TX, TW, VEC, 1024>(p, st);
    }
    if (p.dx) layer_norm_backward_wide_kernel<TX, TW><<<static_cast<unsigned>(p.M), 1024, 0, st>>>(p);
    if (p.part)
        layer_norm_backward_columns_kernel<TX><<<dim3(static_cast<unsigned>((p.N + 255) / 256), static_cast<unsigned>(walking_blocks(p.M, p.N))), 256, 0, st>>>(p);
    return cudaGetLastError();
}

bool known_type(int t) { return t == ATB_F32 || t == ATB_BF16; }
int64_t size_of(int t) { return t == ATB_F32 ? 4 : 2; }
bool aligned_to(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }
bool vec_ok(const void* p, int64_t ld, int type) { return atb::aligned16(p) && ld * size_of(type) % 16 == 0; }

atb_status_t check_common(int64_t M, int64_t N, int x_type, int w_type) {
    if (!known_type(x_type) || !known_type(w_type))
        return atb::fail(ATB_ERR_BAD_ARGUMENT, "x_type=%d, w_type=%d: ATB_F32 or ATB_BF16", x_type, w_type);
    if (M < 0 || N < 0 || M > 0x7FFFFFFFll - 32 || N > (1ll << 30))
        return atb::fail(ATB_ERR_BAD_SHAPE, "need 0 <= M < 2^31 - 32 and 0 <= N <= 2^30 (got %lld, %lld)", (long long)M, (long long)N);
    return ATB_OK;
}

#define ATB_LN_TYPES(CALL)                                                                     \
    if (x_type == ATB_F32 && w_type == ATB_F32) { CALL(float, float); }                        \
    else if (x_type == ATB_F32) { CALL(float, __nv_bfloat16); }                                \
    else if (w_type == ATB_F32) { CALL(__nv_bfloat16, float); }                                \
    else { CALL(__nv_bfloat16, __nv_bfloat16); }

atb_status_t forward(int64_t M, int64_t N, int x_type, const void* X, int64_t ldx, int w_type, const void* W, const void* B,
                     float eps, void* Y, int64_t ldy, uint8_t* exp, float* mean, float* rstd, void* stream) {
    atb::clear_error();
    atb_status_t s = check_common(M, N, x_type, w_type);
    if (s != ATB_OK) return s;
    if (!(eps >= 0.f)) return atb::fail(ATB_ERR_BAD_ARGUMENT, "eps must be >= 0");
    if (exp && N % 8 != 0) return atb::fail(ATB_ERR_BAD_SHAPE, "N=%lld is not a multiple of the block size 8", (long long)N);
    if (M == 0 || N == 0) return ATB_OK;
    if (!X || !Y) return atb::fail(ATB_ERR_NULL_POINTER, "the input and the output must be non-NULL");
    if (ldx < N || (!exp && ldy < N)) return atb::fail(ATB_ERR_BAD_SHAPE, "ldx=%lld and ldy=%lld must be >= N", (long long)ldx, (long long)ldy);
    if (!aligned_to(X, size_of(x_type)) || !aligned_to(W, size_of(w_type)) || !aligned_to(B, size_of(w_type)) ||
        (!exp && !aligned_to(Y, size_of(x_type))) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements");
    const bool vec = N % 8 == 0 && vec_ok(X, ldx, x_type) && atb::aligned16(W) && atb::aligned16(B) && (exp || vec_ok(Y, ldy, x_type));
    if (exp && (!vec || !atb::aligned16(Y) || !atb::aligned16(exp)))
        return atb::fail(ATB_ERR_MISALIGNED, "BFP16 output needs 16-byte aligned pointers and rows of X");
    int sms = 0;
    s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    FwdParams p{M, N, ldx, ldy, exp ? atb::round_up(M, 32) : M, X, W, B, eps, Y, exp, mean, rstd};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
#define ATB_LN_BFP(TX, TW) e = launch_fwd<TX, TW, 8, true>(p, st)
#define ATB_LN_VEC(TX, TW) e = launch_fwd<TX, TW, 8, false>(p, st)
#define ATB_LN_ONE(TX, TW) e = launch_fwd<TX, TW, 1, false>(p, st)
    if (exp) { ATB_LN_TYPES(ATB_LN_BFP) }
    else if (vec) { ATB_LN_TYPES(ATB_LN_VEC) }
    else { ATB_LN_TYPES(ATB_LN_ONE) }
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "layer norm launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

}  // namespace

extern "C" atb_status_t atb_layer_norm(int64_t M, int64_t N, int x_type, const void* X_dev, int64_t ldx, int w_type,
                                       const void* W_dev, const void* B_dev, float eps, void* Y_dev, int64_t ldy,
                                       float* mean_dev, float* rstd_dev, void* stream) {
    return forward(M, N, x_type, X_dev, ldx, w_type, W_dev, B_dev, eps, Y_dev, ldy, nullptr, mean_dev, rstd_dev, stream);
}

extern "C" atb_status_t atb_layer_norm_bfp16(int64_t M, int64_t N, int x_type, const void* X_dev, int64_t ldx, int w_type,
                                             const void* W_dev, const void* B_dev, float eps, int8_t* mant_dev, uint8_t* exp_dev,
                                             float* mean_dev, float* rstd_dev, void* stream) {
    if (M > 0 && N > 0 && !exp_dev) {
        atb::clear_error();
        return atb::fail(ATB_ERR_NULL_POINTER, "the exponent plane must be non-NULL");
    }
    // an empty call passes a non-NULL plane on, so that it is checked as a BFP16 call
    return forward(M, N, x_type, X_dev, ldx, w_type, W_dev, B_dev, eps, mant_dev, N, exp_dev ? exp_dev : reinterpret_cast<uint8_t*>(16),
                   mean_dev, rstd_dev, stream);
}

extern "C" size_t atb_layer_norm_backward_workspace_bytes(int64_t M, int64_t N) {
    if (M < 0 || N < 1) return 0;
    return static_cast<size_t>(partial_sums(M, N)) * 2 * static_cast<size_t>(N) * sizeof(float);
}

extern "C" atb_status_t atb_layer_norm_backward(int64_t M, int64_t N, int x_type, const void* dY_dev, int64_t lddy, const void* X_dev,
                                                int64_t ldx, int w_type, const void* W_dev, const float* mean_dev, const float* rstd_dev,
                                                void* dX_dev, int64_t lddx, void* dW_dev, void* dB_dev,
                                                void* workspace_dev, size_t workspace_bytes, void* stream) {
    atb::clear_error();
    atb_status_t s = check_common(M, N, x_type, w_type);
    if (s != ATB_OK) return s;
    if (N == 0) return ATB_OK;
    const bool sums = dW_dev || dB_dev;
    if (M > 0 && (!dY_dev || !X_dev || !mean_dev || !rstd_dev))
        return atb::fail(ATB_ERR_NULL_POINTER, "dY, X, mean and rstd must be non-NULL");
    if (sums && !workspace_dev) return atb::fail(ATB_ERR_NULL_POINTER, "dW and dB need the workspace");
    if (M > 0 && (ldx < N || lddy < N || (dX_dev && lddx < N)))
        return atb::fail(ATB_ERR_BAD_SHAPE, "lddy=%lld, ldx=%lld and lddx=%lld must be >= N", (long long)lddy, (long long)ldx, (long long)lddx);
    if (!aligned_to(X_dev, size_of(x_type)) || !aligned_to(dY_dev, size_of(x_type)) || !aligned_to(dX_dev, size_of(x_type)) ||
        !aligned_to(W_dev, size_of(w_type)) || !aligned_to(dW_dev, size_of(w_type)) || !aligned_to(dB_dev, size_of(w_type)) ||
        !aligned_to(mean_dev, 4) || !aligned_to(rstd_dev, 4) || !aligned_to(workspace_dev, 16))
        return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements, the workspace to 16 bytes");
    if (sums && workspace_bytes < atb_layer_norm_backward_workspace_bytes(M, N))
        return atb::fail(ATB_ERR_BUFFER_TOO_SMALL, "workspace of %zu bytes is smaller than the %zu needed", workspace_bytes,
                         atb_layer_norm_backward_workspace_bytes(M, N));
    int sms = 0;
    s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    BwdParams p{M, N, lddy, ldx, lddx, dY_dev, X_dev, W_dev, mean_dev, rstd_dev, dX_dev, sums ? static_cast<float*>(workspace_dev) : nullptr};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool vec = N % 8 == 0 && vec_ok(X_dev, ldx, x_type) && vec_ok(dY_dev, lddy, x_type) && atb::aligned16(W_dev) &&
                     (!dX_dev || vec_ok(dX_dev, lddx, x_type));
    cudaError_t e = cudaSuccess;
    if (M > 0 && (dX_dev || sums)) {
#define ATB_LN_BWD_VEC(TX, TW) e = launch_bwd<TX, TW, 8>(p, st)
#define ATB_LN_BWD_ONE(TX, TW) e = launch_bwd<TX, TW, 1>(p, st)
        if (vec) { ATB_LN_TYPES(ATB_LN_BWD_VEC) }
        else { ATB_LN_TYPES(ATB_LN_BWD_ONE) }
    }
    if (e == cudaSuccess && sums) {
        const unsigned blocks = static_cast<unsigned>((2 * N + 31) / 32);
        const int parts = M > 0 ? partial_sums(M, N) : 0;
        const float* const part = p.part;
        if (w_type == ATB_F32)
            e = atb::launch_dependent(layer_norm_backward_sum_kernel<float>, blocks, 32u * kSumWarps, 1u, 0, st, part, parts, N, static_cast<float*>(dW_dev),
                                 static_cast<float*>(dB_dev));
        else
            e = atb::launch_dependent(layer_norm_backward_sum_kernel<__nv_bfloat16>, blocks, 32u * kSumWarps, 1u, 0, st, part, parts, N,
                                 static_cast<__nv_bfloat16*>(dW_dev), static_cast<__nv_bfloat16*>(dB_dev));
    }
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "layer norm backward launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}
