// What the kernels that walk rows share (layer norm, residual norm): how many threads a row takes, loads and stores of groups of elements,
// sums over a row's threads, and rows on their way into shared memory.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <type_traits>

#include "atb_internal.h"
#include "f32x2.cuh"

namespace norm_rows {

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
// The layer norm's backward kernel and both of the residual norm's work on their elements in pairs by the two-wide FP32 instructions, which
// round each half like the scalar ones: 3 to 10 % faster than scalar arithmetic in the former.  (The layer norm's forward kernel,
// with half the arithmetic per byte, was 5 to 15 % slower in this form, and is scalar.)
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


}  // namespace norm_rows
