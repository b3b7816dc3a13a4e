// BF16 x BF16 products with FP32 accumulation for the gated feed-forward block, the linear cross entropy and the linear layer (sm_100a).
//
// C = A x B with either operand stored along K or across it (the three layouts that a layer's forward and backward
// products need), on tcgen05 with the accumulator in tensor memory, and epilogues that finish the operator's own
// arithmetic on the accumulator before anything is written.
//
// One persistent CTA per SM, or a pair of CTAs (cta_group::2) per two SMs.  Warp 0 brings the operand tiles in by TMA
// (128-byte swizzle, 64 x 64 boxes: 32 KB per CTA and K-step of 64 in both forms), one lane of warp 1 issues the
// UMMAs, eight warps run the epilogue.  The accumulator is held twice, so that a tile's epilogue runs beside the next
// tile's K loop.
//   pair    256 x 256 tile: each CTA loads its 128 rows of A and half of the columns of B and holds 128 x 256 of C
//   single  128 x 128 tile: four times as many tiles for outputs that would leave most of the SMs idle; for the head of a few
//           rows, which is bound by reading W, the tile's width is what deals the words out evenly (16 to 128)
// Up to three products that do not depend on one another (the gradients of a layer's input and weights) share a launch:
// their tiles are dealt out as one list, so that one product's last wave is filled by the next one's tiles.  A product
// of few tiles is cut along K into ranges whose FP32 sums a second kernel joins.
// Bound by the tensor cores where there are tiles enough, at 4096 x 4096 x 10944 and 4096 x 65536 x 2048 (of a measured 1653
// TFLOP/s for a lone library product): both projections with the activation and g, u, h written 461 us, 1593 TFLOP/s (g and u in
// FP32: 486 us, 1512); gated backward epilogue 257 us, 1429 TFLOP/s (273 us, 1345; 688 tiles are 9.3 rounds of 74 pairs); the gradients
// behind it in one launch 1196 us, 1535 TFLOP/s under the power cap; row statistics of the head 666 us, 1650
// TFLOP/s, tensor pipe 98 % busy; softmax gradient 701 us, 1568 TFLOP/s, 93 %.  Bound by memory where rows are few: the head of 60 rows over
// 131072 x 2048 words 85 us, 6.35 TB/s.  In between by fill, drain and launch, 4 us per kernel.
// Tried and dropped: plain coalesced stores instead of TMA stores out of the epilogues' boxes (level, +-1 %), two boxes per warp
// and five stages (level).
// Every wait is bounded (see atb_gemm_device.cuh).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "atb_bf16_mm.h"
#include "atb_gemm_device.cuh"
#include "dependent_launch.cuh"
#include "glu.cuh"

namespace {

using namespace glu;
using atb::kMmGroup;

__device__ unsigned int g_mm_error_flag = 0;

constexpr int kMmKStep = 64;
constexpr uint32_t kMmBoxBytes = 64 * 128;              // 64 rows of 64 bf16
constexpr uint32_t kMmTileBytes = 2 * kMmBoxBytes;      // a CTA's part of A, or of B, for one K-step
constexpr int kMmEpiWarps = 8, kMmFirstEpiWarp = 2;
constexpr int kMmThreads = (kMmFirstEpiWarp + kMmEpiWarps) * 32;

// One product of a launch, as the kernel sees it.
struct MmJob {
    int64_t M, N;
    int a_mn, b_mn;                    // operands stored across K
    int m_tiles, n_tiles, n_segs;      // n_tiles: of one segment
    int k_steps0, k_steps;             // steps of the first K segment, of both
    int splits;                        // the K loop is cut into this many ranges, units of work of their own
    int a_rows;                        // rows of A that a CTA loads: 128, or what there is of a K-major A of 64 rows and less
    int first_item;                    // of this product in the launch's list of (range, tile)
    int fp32, add;                     // C in FP32 (the sums of a range, rows split * split_rows on; or C32), added to it
    int64_t split_rows;
    const float* factor;               // of C, or NULL
};

struct MmParams {
    MmJob job[kMmGroup];
    int n_jobs, items;
    int stages, tile_n;                    // stages of the operand ring, of a_bytes + b_bytes each
    uint32_t a_bytes, b_bytes;
    unsigned int* error_flag;
    int act, save;
    const int64_t* labels;
    int64_t ignore_index, col0;
    float2* stats;
    int64_t stats_ld;
    float* label_logit;
    const float *lse, *scale;
    float* unit;
    int64_t rows;                          // kMmDlogits: of the product
    bool first;
    void* dl;                              // kMmDlogits, tiles of any width
    int64_t dl_ld;
    const void* bias;                      // kMmLinear
    int bias32, residual, kept;            // kept: 0, kKeptBf16 or kKeptF32
};

constexpr int kKeptBf16 = 1, kKeptF32 = 2;      // type of the sums before the activation that kMmLinear leaves

// Tensor maps: product j has A at a[2 j], a[2 j + 1] (K segments), B and C alike (segments).  The epilogues of a single product
// use c[0 .. 3]: h, g, u; dg, du, g, u; dl; y, z, r.
template <int JOBS>
struct MmMaps {
    CUtensorMap a[2 * JOBS], b[2 * JOBS], c[JOBS == 1 ? 4 : 2 * JOBS];
};

struct MmJoinJob {
    int64_t M, N, cols, split_rows, first;       // first: of this product in the list of groups of eight columns
    int n_segs, splits, add;
    const float *src, *factor;
    void* C[3];
    int64_t ldc[3];
    float* C32;
};
struct MmJoin {
    MmJoinJob job[kMmGroup];
    int n_jobs, act;
    int64_t all;
    const void *G, *U;
    const void *bias, *R;                        // kMmLinear
    int64_t ldr;
    int bias32, z32;
};

constexpr int kMmPlain = 100;          // kMmStore and kMmAccumulate: one kernel

template <bool PAIR, int EPI>
struct MmCfg {
    static constexpr int JOBS = EPI == kMmPlain ? kMmGroup : 1;
    static constexpr int BN = PAIR ? 256 : 128;             // accumulator columns
    static constexpr int TILE_M = PAIR ? 256 : 128;
    static constexpr bool DUAL = EPI == atb::kMmGlu;        // half of the columns from B[0], half from B[1]
    static constexpr int TILE_N = DUAL ? BN / 2 : BN;       // columns of C per tile
    static constexpr int COLS = DUAL ? 64 : BN / 2;         // columns of C of an epilogue warp (a 64-column tile has one group)
    static constexpr int BOXES = (EPI == atb::kMmGlu || EPI == atb::kMmGluBackward || EPI == atb::kMmLinear) ? 2 : 1;   // staging boxes of a warp
    static constexpr int BOX_BARS = EPI == atb::kMmLinear ? 2 : 1;       // barriers of the loads into them
    static constexpr uint32_t STAGE_BYTES = 2 * kMmTileBytes;
    // Ring of operand stages: 5 or 6, more (single CTAs) where A is a few rows and a stage little more than its B tile
    static constexpr uint32_t BOX_OFF = (BOXES == 2 ? 5 : 6) * STAGE_BYTES;
    static constexpr int MOST_STAGES = PAIR ? BOX_OFF / STAGE_BYTES : 32;
    // The tile's width is the launch's (MmParams::tile_n)
    static constexpr bool ANY_WIDTH = !PAIR && (EPI == atb::kMmRowStats || EPI == atb::kMmDlogits);
    static constexpr uint32_t BAR_OFF = BOX_OFF + kMmEpiWarps * BOXES * kEpilogueBoxBytes;
    static constexpr uint32_t SMEM_BYTES = 1024 + BAR_OFF + 8 * (2 * MOST_STAGES + 4 + kMmEpiWarps * BOX_BARS) + 16;
    static_assert(SMEM_BYTES <= kSmemBudget, "shared memory");
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 b2 = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b2);
}

__device__ __forceinline__ float2 unpack_bf16(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }

// h = act(g) u of two neighbours, packed.
template <int ACT>
__device__ __forceinline__ uint32_t glu_pair(float2 g, float2 u) {
    float2 a, slope;
    act_value_slope<ACT>(g, a, slope);
    const float2 h = f32x2::mul2(a, u);
    return pack_bf16(h.x, h.y);
}
// dg = dh u act'(g) and du = dh act(g) of two neighbours, packed.
template <int ACT>
__device__ __forceinline__ void glu_backward_pair(float2 g, float2 u, float2 dh, uint32_t& dg, uint32_t& du) {
    float2 a, slope;
    act_value_slope<ACT>(g, a, slope);
    const float2 x = f32x2::mul2(f32x2::mul2(dh, u), slope), y = f32x2::mul2(dh, a);
    dg = pack_bf16(x.x, x.y);
    du = pack_bf16(y.x, y.y);
}

// A warp's staging boxes of 32 rows x 64 bf16 or 32 fp32 (128-byte swizzle), used in turn; each leaves by a TMA store, or is
// added to memory by one, which clips at the edges of the output.
template <int BOXES>
struct BoxWriter {
    uint32_t base, bar;                    // the boxes; barrier of the loads into them
    int lane, next = 0;
    uint32_t phase = 0;
    __device__ BoxWriter(uint32_t b, uint32_t bar_, int l) : base(b), bar(bar_), lane(l) {}
    __device__ __forceinline__ void put(const CUtensorMap* map, const uint32_t (&o)[32], int64_t col, int64_t row0, bool inside, bool add = false) {
        if (lane == 0) tma_store_wait_read<BOXES - 1>();       // the store that last used this box has read it
        __syncwarp();
        write(next, o);
        if (lane == 0) {
            if (inside) {
                if (add) tma_reduce_add_2d(map, box(next), static_cast<int>(col), static_cast<int>(row0));
                else tma_store_2d(map, box(next), static_cast<int>(col), static_cast<int>(row0));
            }
            tma_store_commit();                                // an empty group keeps the count of groups per box
        }
        next = next + 1 == BOXES ? 0 : next + 1;
    }
    // By plain stores of 16-byte pieces, 8 lanes to a row: rows below M, pieces that start below column N.
    __device__ __forceinline__ void put_pieces(__nv_bfloat16* C, int64_t ld, const uint32_t (&o)[32], int64_t col, int64_t row0, int64_t M, int64_t N) const {
        __syncwarp();                      // the box's last contents have been read
        write(0, o);
        __syncwarp();
        const int och = lane & 7, orow = lane >> 3;
        const int64_t at = col + och * 8, rows_left = M - row0 - orow;
        __nv_bfloat16* dst = C + (row0 + orow) * ld + at;
        const uint32_t src = box(0) + orow * 128;
        if (at >= N) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint4 v;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                         : "r"(src + i * 512 + ((static_cast<uint32_t>(och) ^ static_cast<uint32_t>((4 * i + orow) & 7)) << 4)) : "memory");
            if (4 * i < rows_left) *reinterpret_cast<uint4*>(dst + 4 * i * ld) = v;
        }
    }
    // The other direction: 64 bf16 or 32 FP32 columns of two inputs into the two boxes, and what becomes of them out of the same boxes.
    __device__ __forceinline__ void fetch(const CUtensorMap* m0, const CUtensorMap* m1, int64_t col, int64_t row0) {
        if (lane == 0) {
            tma_store_wait_read<0>();
            mbar_arrive_expect_tx(bar, 2 * kEpilogueBoxBytes);
            tma_load_2d(box(0), m0, static_cast<int>(col), static_cast<int>(row0), bar);
            tma_load_2d(box(1), m1, static_cast<int>(col), static_cast<int>(row0), bar);
        }
        __syncwarp();
    }
    __device__ __forceinline__ bool fetched(const Ctx& cx) {
        const bool ok = wait_bar(cx, bar, phase, 0x202);
        phase ^= 1u;
        next = 0;
        return ok;
    }
    // One input into box b, whose last store has been read (barrier bar + 8 b; bit b of `phase`).
    __device__ __forceinline__ void fetch_box(int b, const CUtensorMap* m, int64_t col, int64_t row0) {
        if (lane == 0) {
            tma_store_wait_read<0>();
            mbar_arrive_expect_tx(bar + 8 * b, kEpilogueBoxBytes);
            tma_load_2d(box(b), m, static_cast<int>(col), static_cast<int>(row0), bar + 8 * b);
        }
        __syncwarp();
    }
    __device__ __forceinline__ bool box_fetched(const Ctx& cx, int b) {
        const bool ok = wait_bar(cx, bar + 8 * b, (phase >> b) & 1u, 0x203);
        phase ^= 1u << b;
        next = b;
        return ok;
    }
    // Columns 32 part .. + 31 of this lane's row (packed bf16).
    __device__ __forceinline__ void read(int b, int part, uint32_t (&v)[16]) const {
        const uint32_t row = box(b) + lane * 128, sw = lane & 7;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[4 * j]), "=r"(v[4 * j + 1]), "=r"(v[4 * j + 2]), "=r"(v[4 * j + 3])
                         : "r"(row + ((static_cast<uint32_t>(4 * part + j) ^ sw) << 4)) : "memory");
    }
    // This lane's row, 32 FP32 columns.
    __device__ __forceinline__ void read_row(int b, uint32_t (&v)[32]) const {
        const uint32_t row = box(b) + lane * 128, sw = lane & 7;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[4 * j]), "=r"(v[4 * j + 1]), "=r"(v[4 * j + 2]), "=r"(v[4 * j + 3])
                         : "r"(row + ((static_cast<uint32_t>(j) ^ sw) << 4)) : "memory");
    }
    // Between reads of the boxes and the next fetch, where no write stands between.
    __device__ __forceinline__ void rows_read() const {
        fence_proxy_async_smem();
        __syncwarp();
    }
    __device__ __forceinline__ void put_in_place(const CUtensorMap* map, const uint32_t (&o)[32], int64_t col, int64_t row0) {
        write(next, o);
        if (lane == 0) {
            tma_store_2d(map, box(next), static_cast<int>(col), static_cast<int>(row0));
            tma_store_commit();
        }
        ++next;
    }
private:
    __device__ __forceinline__ uint32_t box(int b) const { return base + b * kEpilogueBoxBytes; }
    __device__ __forceinline__ void write(int b, const uint32_t (&o)[32]) const {
        const uint32_t row = box(b) + lane * 128, sw = lane & 7;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row + ((static_cast<uint32_t>(j) ^ sw) << 4)),
                         "r"(o[4 * j]), "r"(o[4 * j + 1]), "r"(o[4 * j + 2]), "r"(o[4 * j + 3]) : "memory");
        fence_proxy_async_smem();
        __syncwarp();
    }
};

// The unit that dl is held in.  Rounded to bf16 as it is, a scale of 1 / 255 (a mean over 255 rows) would put the same 0.4 % on every
// row's label, and so on dx and dW; in units of the largest scale, equal scales are exactly 1, and the products behind dl
// multiply by the unit in FP32.  Every CTA finds it for itself while its first tile is on its way (M = 8192: 32 rows per thread),
// all alike; the first launch of a call leaves it for the launches behind.  Infinite and NaN scales stay their rows' own affair.
__device__ __forceinline__ float mm_unit(const MmParams& p, uint32_t boxes, uint32_t box_stride, int e, int lane) {
    if (!p.first) return *p.unit;
    float most = 0.f;
#pragma unroll 8
    for (int64_t m = e * 32 + lane; m < p.rows; m += kMmEpiWarps * 32) {
        const float a = fabsf(p.scale[m]);
        if (p.labels[m] != p.ignore_index && a <= 3.402823466e38f) most = fmaxf(most, a);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    // through the first word of each warp's staging boxes, which hold nothing yet
    if (lane == 0) asm volatile("st.shared.f32 [%0], %1;" ::"r"(boxes + e * box_stride), "f"(most) : "memory");
    asm volatile("bar.sync 1, %0;" ::"n"(kMmEpiWarps * 32) : "memory");
#pragma unroll
    for (int w = 0; w < kMmEpiWarps; ++w) {
        float v;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(boxes + w * box_stride) : "memory");
        most = fmaxf(most, v);
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kMmEpiWarps * 32) : "memory");
    if (most == 0.f) most = 1.f;
    if (blockIdx.x == 0 && e == 0 && lane == 0) *p.unit = most;
    return most;
}

// ------------------------------------------------------------------------------------------ the linear layer's epilogue
// Values of N columns from col on, for all lanes alike; 0 past the last column and where there is no bias.
template <int COUNT>
__device__ __forceinline__ void load_bias(const void* bias, int bias32, int64_t col, int64_t N, float (&b)[COUNT]) {
#pragma unroll
    for (int e = 0; e < COUNT; ++e) b[e] = 0.f;
    if (!bias) return;
    if (bias32) {
        const float4* src = reinterpret_cast<const float4*>(static_cast<const float*>(bias) + col);
#pragma unroll
        for (int j = 0; j < COUNT / 4; ++j)
            if (col + 4 * j < N) {
                const float4 v = __ldg(src + j);
                b[4 * j] = v.x; b[4 * j + 1] = v.y; b[4 * j + 2] = v.z; b[4 * j + 3] = v.w;
            }
    } else {
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(bias) + col);
#pragma unroll
        for (int j = 0; j < COUNT / 8; ++j)
            if (col + 8 * j < N) {
                const uint4 v = __ldg(src + j);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = unpack_bf16(w[e]);
                    b[8 * j + 2 * e] = f.x; b[8 * j + 2 * e + 1] = f.y;
                }
            }
    }
}

// act(z + bias) + residual of COLS columns of 32 rows.  A piece is a box: 64 bf16 columns or 32 FP32 ones (Y32).  The residual arrives
// in the boxes in turn, the first two pieces fetched before the accumulator was waited for (linear_fetch), and the result
// takes its place.  Where the sums before the activation are kept too, those leave through the boxes first, 64 columns at a time, the
// residual is fetched piece by piece, and the accumulator is read a second time: nothing has to stay in registers in between.
template <class C, bool Y32>
__device__ __forceinline__ void linear_fetch(const MmMaps<1>& tm, const MmParams& p, const MmJob& jb, BoxWriter<2>& out, int64_t row0, int64_t col0) {
    constexpr int PIECE = Y32 ? 32 : 64;
    if (!p.residual || p.kept || row0 >= jb.M) return;
#pragma unroll
    for (int b = 0; b < 2; ++b)
        if (b * PIECE < C::COLS && col0 + b * PIECE < jb.N) out.fetch_box(b, &tm.c[2], col0 + b * PIECE, row0);
}
// A warp's bias: lane i has columns i, 32 + i, ... of its own, loaded while the accumulator is waited for.  (Loaded where it is used, a few columns
// at a time for all lanes alike, it cost a prompt of 509 rows 3.5 of 22 us.)
template <class C>
struct LinearBias {
    float v[C::COLS / 32];
    __device__ __forceinline__ LinearBias(const MmParams& p, const MmJob& jb, int64_t col0, int lane) {
#pragma unroll
        for (int i = 0; i < C::COLS / 32; ++i) {
            const int64_t col = col0 + 32 * i + lane;
            v[i] = 0.f;
            if (p.bias && col < jb.N)
                v[i] = p.bias32 ? __ldg(static_cast<const float*>(p.bias) + col)
                                : __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const uint16_t*>(p.bias) + col)) << 16);
        }
    }
    // of this lane's column of the 32 from column c of the warp's on
    __device__ __forceinline__ float at(int c) const {
        float b = v[0];
#pragma unroll
        for (int i = 1; i < C::COLS / 32; ++i) b = c == 32 * i ? v[i] : b;
        return b;
    }
};

template <class C, bool Y32>
__device__ __forceinline__ void linear_epilogue(const MmMaps<1>& tm, const MmParams& p, const MmJob& jb, BoxWriter<2>& out, const LinearBias<C>& bias, uint32_t t_addr,
                                                int64_t row0, int64_t col0, int lane, const Ctx& cx) {
    constexpr int PIECE = Y32 ? 32 : 64;
    if (row0 >= jb.M) return;
    const bool in_place = p.residual && !p.kept;
    // z of 32 columns
    const auto sums = [&](int c, uint32_t (&v)[32]) {
        tmem_ld_32x32b_x32(t_addr + c, v);
        tmem_ld_wait_for(v);
        if (!p.bias) return;
        const float mine = bias.at(c);
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) + __shfl_sync(0xFFFFFFFFu, mine, e));
    };
    with_linear_act(p.act, [&](auto act) {
#pragma unroll 1
        for (int c = 0; c < C::COLS && col0 + c < jb.N; c += PIECE) {
            const int64_t col = col0 + c;
            const int b = in_place ? (c / PIECE) & 1 : 0;
            uint32_t v[32], o[32];
            if (p.kept && !(c & 32)) {     // columns past the last one are clipped
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    sums(c + 32 * part, v);
                    if (p.kept == kKeptF32) {
                        out.put(&tm.c[1], v, col + 32 * part, row0, col + 32 * part < jb.N);
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[16 * part + e] = pack_bf16(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
                    }
                }
                if (p.kept == kKeptBf16) out.put(&tm.c[1], o, col, row0, true);
            }
            if (p.residual) {
                if (!in_place) out.fetch_box(0, &tm.c[2], col, row0);
                if (!out.box_fetched(cx, b)) return;
            }
            if constexpr (Y32) {
                sums(c, v);
                if (p.residual) out.read_row(b, o);
                else
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0u;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float2 a = f32x2::add2(act_value<act.value>(make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]))),
                                                 make_float2(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1])));
                    o[2 * e] = __float_as_uint(a.x);
                    o[2 * e + 1] = __float_as_uint(a.y);
                }
            } else {
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t r[16];
                    sums(c + 32 * part, v);
                    if (p.residual) out.read(b, part, r);
                    else
#pragma unroll
                        for (int e = 0; e < 16; ++e) r[e] = 0u;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float2 a = f32x2::add2(act_value<act.value>(make_float2(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]))), unpack_bf16(r[e]));
                        o[16 * part + e] = pack_bf16(a.x, a.y);
                    }
                }
            }
            if (in_place) {
                out.put_in_place(&tm.c[0], o, col, row0);
                // the piece after the next one, into the box that this one leaves
                if (c + 2 * PIECE < C::COLS && col + 2 * PIECE < jb.N) out.fetch_box(b, &tm.c[2], col + 2 * PIECE, row0);
            } else {
                if (p.residual) out.rows_read();
                out.put(&tm.c[0], o, col, row0, true);
            }
        }
    });
}

// ------------------------------------------------------------------------------------------ epilogue of one warp
// Rows row0 .. row0 + 31 (one per lane); t_addr: the warp's lanes of the tile's accumulator, column 0; half: which of
// the tile's column groups this warp has, of `cols` columns; col0: first column of the tile in C.
template <class C, int EPI, bool KEEP32>
__device__ __forceinline__ void mm_epilogue(const MmMaps<C::JOBS>& tm, const MmParams& p, const MmJob& jb, int c_map, BoxWriter<C::BOXES>& out,
                                            uint32_t t_addr, int half, int64_t row0, int64_t col0, int cols, int split, float unit, int lane, const Ctx& cx) {
    const int64_t row = row0 + lane;
    const bool row_in = row < jb.M, warp_in = row0 < jb.M;
    const int64_t slot = C::ANY_WIDTH ? col0 / p.tile_n * (p.tile_n > C::COLS ? 2 : 1) + half : col0 / C::COLS + half;     // kMmRowStats
    col0 += half * C::COLS;
    t_addr += half * C::COLS;
    (void)slot;
    if constexpr (EPI == kMmPlain) {
        const float factor = jb.factor ? *jb.factor : 1.f;
        if (!jb.fp32) {
#pragma unroll 1
            for (int c = 0; c < C::COLS; c += 64) {
                uint32_t v[32], w[32], o[32];
                tmem_ld_32x32b_x32(t_addr + c, v);
                tmem_ld_32x32b_x32(t_addr + c + 32, w);
                tmem_ld_wait_for(v);
                tmem_ld_wait_for(w);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    o[e] = pack_bf16(factor * __uint_as_float(v[2 * e]), factor * __uint_as_float(v[2 * e + 1]));
                    o[16 + e] = pack_bf16(factor * __uint_as_float(w[2 * e]), factor * __uint_as_float(w[2 * e + 1]));
                }
                out.put(&tm.c[c_map], o, col0 + c, row0, warp_in && col0 + c < jb.N);
            }
        } else {
#pragma unroll 1
            for (int c = 0; c < C::COLS; c += 32) {
                uint32_t v[32];
                tmem_ld_32x32b_x32(t_addr + c, v);
                tmem_ld_wait_for(v);
#pragma unroll
                for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(factor * __uint_as_float(v[e]));
                out.put(&tm.c[c_map], v, col0 + c, split * jb.split_rows + row0, warp_in && col0 + c < jb.N, jb.add);
            }
        }
    } else if constexpr (EPI == atb::kMmGlu) {
        // accumulator columns 0 .. TILE_N - 1 hold g, the next TILE_N hold u
        const bool inside = warp_in && col0 < jb.N;
        with_act(p.act, [&](auto act) {
            uint32_t h[32];
            // 32 columns of both and h of them
            const auto part_of = [&](int part, uint32_t (&g)[32], uint32_t (&u)[32]) {
                tmem_ld_32x32b_x32(t_addr + 32 * part, g);
                tmem_ld_32x32b_x32(t_addr + C::TILE_N + 32 * part, u);
                tmem_ld_wait_for(g);
                tmem_ld_wait_for(u);
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    h[16 * part + e] = glu_pair<act.value>(make_float2(__uint_as_float(g[2 * e]), __uint_as_float(g[2 * e + 1])),
                                                           make_float2(__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1])));
            };
            if constexpr (KEEP32) {
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t g[32], u[32];
                    part_of(part, g, u);
                    out.put(&tm.c[1], g, col0 + 32 * part, row0, warp_in && col0 + 32 * part < jb.N);
                    out.put(&tm.c[2], u, col0 + 32 * part, row0, warp_in && col0 + 32 * part < jb.N);
                }
                out.put(&tm.c[0], h, col0, row0, inside);
            } else {
                uint32_t og[32], ou[32];
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t g[32], u[32];
                    part_of(part, g, u);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        og[16 * part + e] = pack_bf16(__uint_as_float(g[2 * e]), __uint_as_float(g[2 * e + 1]));
                        ou[16 * part + e] = pack_bf16(__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1]));
                    }
                }
                out.put(&tm.c[0], h, col0, row0, inside);
                if (p.save) {
                    out.put(&tm.c[1], og, col0, row0, inside);
                    out.put(&tm.c[2], ou, col0, row0, inside);
                }
            }
        });
    } else if constexpr (EPI == atb::kMmGluBackward) {
        // g and u of 64 columns (of 32 twice, where they are FP32) arrive in the two boxes, the first ones fetched before the accumulator
        // was waited for; a lane replaces its row in them by dg and du
        if (!warp_in) return;
        with_act(p.act, [&](auto act) {
            if constexpr (KEEP32) {
#pragma unroll 1
                for (int c = 0; c < C::COLS && col0 + c < jb.N; c += 64) {
                    if (c > 0) out.fetch(&tm.c[2], &tm.c[3], col0 + c, row0);
                    uint32_t og[32], ou[32];
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        uint32_t dh[32], g[32], u[32];
                        if (!out.fetched(cx)) return;
                        out.read_row(0, g);
                        out.read_row(1, u);
                        if (part == 0) {       // columns past the last one are zeros
                            out.rows_read();
                            out.fetch(&tm.c[2], &tm.c[3], col0 + c + 32, row0);
                        }
                        tmem_ld_32x32b_x32(t_addr + c + 32 * part, dh);
                        tmem_ld_wait_for(dh);
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            glu_backward_pair<act.value>(make_float2(__uint_as_float(g[2 * e]), __uint_as_float(g[2 * e + 1])),
                                                         make_float2(__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1])),
                                                         make_float2(__uint_as_float(dh[2 * e]), __uint_as_float(dh[2 * e + 1])),
                                                         og[16 * part + e], ou[16 * part + e]);
                    }
                    out.put_in_place(&tm.c[0], og, col0 + c, row0);
                    out.put_in_place(&tm.c[1], ou, col0 + c, row0);
                }
            } else {
#pragma unroll 1
                for (int c = 0; c < C::COLS && col0 + c < jb.N; c += 64) {
                    if (c > 0) out.fetch(&tm.c[2], &tm.c[3], col0 + c, row0);
                    if (!out.fetched(cx)) return;
                    uint32_t og[32], ou[32];
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        uint32_t dh[32], g[16], u[16];
                        tmem_ld_32x32b_x32(t_addr + c + 32 * part, dh);
                        out.read(0, part, g);
                        out.read(1, part, u);
                        tmem_ld_wait_for(dh);
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            glu_backward_pair<act.value>(unpack_bf16(g[e]), unpack_bf16(u[e]), make_float2(__uint_as_float(dh[2 * e]), __uint_as_float(dh[2 * e + 1])),
                                                         og[16 * part + e], ou[16 * part + e]);
                    }
                    out.put_in_place(&tm.c[0], og, col0 + c, row0);
                    out.put_in_place(&tm.c[1], ou, col0 + c, row0);
                }
            }
        });
    } else if constexpr (EPI == atb::kMmRowStats) {
        // columns of this warp inside the vocabulary; the label's, counted from the first
        const int mine = static_cast<int>(min(static_cast<int64_t>(cols), jb.N - col0));
        int64_t label = -1;
        if (row_in) label = p.labels[row] - p.col0 - col0;
        float m = -INFINITY, s = 0.f;
#pragma unroll 1
        for (int c = 0; c < mine; c += 32) {
            uint32_t v[32];
            tmem_ld_32x32b_x32(t_addr + c, v);
            tmem_ld_wait_for(v);
            const int left = mine - c;
            const bool here = label >= c && label < c + 32 && label - c < left;
            if (__any_sync(0xFFFFFFFFu, here)) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (here && label - c == e) p.label_logit[row] = __uint_as_float(v[e]);
            }
            if (left < 32) {
#pragma unroll
                for (int e = 0; e < 32; ++e)
                    if (e >= left) v[e] = 0xFF800000u;         // -inf
            }
            float top = m;
#pragma unroll
            for (int e = 0; e < 32; ++e) top = fmaxf(top, __uint_as_float(v[e]));
            const float ref = top == -INFINITY ? 0.f : top;    // nothing but -inf so far: every term is 0
            // the difference is taken first: exact near the maximum, where the terms that count are
            s *= exp2_fast((m - ref) * kLog2e);
#pragma unroll
            for (int e = 0; e < 32; ++e) s += exp2_fast((__uint_as_float(v[e]) - ref) * kLog2e);
            m = top;
        }
        if (row_in && mine > 0) p.stats[row * p.stats_ld + slot] = make_float2(m, s);
    } else {
        int64_t label = -1;
        float lse = 0.f, scale = 0.f;
        bool counts = false;
        if (row_in) {
            const int64_t l = p.labels[row];
            counts = l != p.ignore_index;
            label = l - p.col0 - col0;
            lse = p.lse[row];
            scale = p.scale[row] / unit;
        }
#pragma unroll 1
        for (int c = 0; c < cols; c += 64) {
            uint32_t o[32];
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                uint32_t v[32];
                tmem_ld_32x32b_x32(t_addr + c + 32 * part, v);
                tmem_ld_wait_for(v);
                const int64_t at = label - (c + 32 * part);
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const float prob = exp2_fast((__uint_as_float(v[e]) - lse) * kLog2e);
                    const float d = (at == e ? prob - 1.f : prob) * scale;
                    v[e] = counts ? __float_as_uint(d) : 0u;   // an ignored row is 0 whatever its logits are
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) o[16 * part + e] = pack_bf16(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
            }
            // a tile of any width ends inside a box, which a TMA store would write beyond it; the words of dl's rows past the piece's
            // end are room for whole 16-byte pieces
            if constexpr (C::ANY_WIDTH) out.put_pieces(static_cast<__nv_bfloat16*>(p.dl), p.dl_ld, o, col0 + c, row0, jb.M, min(col0 + cols, jb.N));
            else out.put(&tm.c[0], o, col0 + c, row0, warp_in && col0 + c < jb.N);
        }
    }
}

// ------------------------------------------------------------------------------------------ kernel
template <bool PAIR>
__device__ __forceinline__ void mm_tma(uint32_t dst, const CUtensorMap* m, int x, int y, uint32_t bar) {
    if constexpr (PAIR) tma_load_2d_pair(dst, m, x, y, bar);
    else tma_load_2d(dst, m, x, y, bar);
}
// 128 rows (or columns) from mn0 on, K-elements k0 .. k0 + 63: two boxes.
template <bool PAIR>
__device__ __forceinline__ void mm_load(uint32_t dst, const CUtensorMap* m0, const CUtensorMap* m1, bool mn_major, int mn0, int mn1, int k0, uint32_t bar) {
    mm_tma<PAIR>(dst, m0, mn_major ? mn0 : k0, mn_major ? k0 : mn0, bar);
    mm_tma<PAIR>(dst + kMmBoxBytes, m1, mn_major ? mn1 : k0, mn_major ? k0 : mn1, bar);
}
// Descriptor of a 128-wide operand tile (see umma_smem_desc_sw128); 16 K-elements on it grows by mm_desc_step.
__device__ __forceinline__ uint64_t mm_desc(uint32_t tile, bool mn_major) { return umma_smem_desc_sw128(tile, mn_major ? kMmBoxBytes : 16u, 1024); }
__device__ __forceinline__ uint32_t mm_desc_step(bool mn_major) { return (mn_major ? 2048u : 32u) >> 4; }

// One unit of work: a tile of a product and a range of its K-steps.
struct MmItem {
    int job, mt, nt, seg, split, k_begin, k_end;
};
// Place in the list of the it-th item of this CTA or pair: dealt out to and fro, so that the units that get the longer items
// of one round get the shorter ones of the next.
template <bool PAIR>
__device__ __forceinline__ int mm_item_at(int it) {
    const int unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, units = PAIR ? gridDim.x >> 1 : gridDim.x;
    return it * units + ((it & 1) ? units - 1 - unit : unit);
}
template <int JOBS>
__device__ __forceinline__ MmItem mm_item(const MmParams& p, int item) {
    MmItem w;
    w.job = 0;
    if constexpr (JOBS > 1)
        while (w.job + 1 < p.n_jobs && item >= p.job[w.job + 1].first_item) ++w.job;
    const MmJob& jb = p.job[w.job];
    const int all_n = jb.n_tiles * jb.n_segs, tiles = jb.m_tiles * all_n;
    item -= jb.first_item;
    w.split = item / tiles;
    tile_coords<8>(item - w.split * tiles, jb.m_tiles, all_n, w.mt, w.nt);
    w.seg = w.nt >= jb.n_tiles ? 1 : 0;
    w.nt -= w.seg * jb.n_tiles;
    w.k_begin = static_cast<int>(static_cast<int64_t>(jb.k_steps) * w.split / jb.splits);
    w.k_end = static_cast<int>(static_cast<int64_t>(jb.k_steps) * (w.split + 1) / jb.splits);
    return w;
}

// KEEP32 (kMmGlu, kMmGluBackward): g and u are FP32 in memory.  A kernel of its own: with both forms in one, their code, which a launch
// finds in no cache after other kernels, took 6 us more of each launch.
template <bool PAIR, int EPI, bool KEEP32>
__global__ void __launch_bounds__(kMmThreads, 1)
bf16_mm_kernel(const __grid_constant__ MmMaps<MmCfg<PAIR, EPI>::JOBS> tm, const __grid_constant__ MmParams p) {
    using C = MmCfg<PAIR, EPI>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar_base = smem_base + C::BAR_OFF;
    const uint32_t full = bar_base, empty = full + 8 * C::MOST_STAGES;
    const uint32_t acc_full = empty + 8 * C::MOST_STAGES, acc_empty = acc_full + 16, box_bar = acc_empty + 16;
    const uint32_t misc = box_bar + 8 * kMmEpiWarps * C::BOX_BARS;       // [0]: TMEM base, [1]: abort flag
    volatile uint32_t* const misc_gen = reinterpret_cast<volatile uint32_t*>(smem_raw + (misc - smem_u32(smem_raw)));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    Ctx cx{misc_gen + 1, p.error_flag};

    if (threadIdx.x == 0) {
        for (int i = 0; i < C::MOST_STAGES; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + 8 * i, 1); mbar_init(acc_empty + 8 * i, kMmEpiWarps * (PAIR ? 2 : 1)); }
        for (int i = 0; i < kMmEpiWarps * C::BOX_BARS; ++i) mbar_init(box_bar + 8 * i, 1);
        misc_gen[1] = 0u;
        fence_mbar_init();
        prefetch_tensormap(&tm.a[0]);
        prefetch_tensormap(&tm.b[0]);
        prefetch_tensormap(&tm.c[0]);
    }
    if (warp == 1) {
        if constexpr (PAIR) { tmem_alloc_pair(misc, 2 * C::BN); tmem_relinquish_pair(); }
        else { tmem_alloc(misc, 2 * C::BN); tmem_relinquish(); }
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();                // the peer's barriers exist before anything arrives on them
    tcgen05_fence_after_sync();
    const uint32_t tmem_base = misc_gen[0];
    const int stages = PAIR ? C::MOST_STAGES : p.stages;
    const uint32_t a_bytes = PAIR ? kMmTileBytes : p.a_bytes, b_bytes = C::ANY_WIDTH ? p.b_bytes : kMmTileBytes, stage_bytes = a_bytes + b_bytes;
    const int tile_n = C::ANY_WIDTH ? p.tile_n : C::TILE_N;
    // what a kernel before this one on the stream wrote may be read from here on
    grid_dependency_wait();
    grid_dependency_launch();

    if (warp == 0) {
        // ================================ TMA producer ================================
        if (elect_one()) {
            Ring r;
            bool ok = true;
            int it = 0;
            for (int item; ok && (item = mm_item_at<PAIR>(it)) < p.items; ++it) {
                const MmItem w = mm_item<C::JOBS>(p, item);
                const MmJob& jb = p.job[w.job];
                const bool a_mn = jb.a_mn, b_mn = jb.b_mn;
                const CUtensorMap* const ta = &tm.a[2 * w.job];
                const CUtensorMap* const tb = &tm.b[2 * w.job];
                const int m0 = w.mt * C::TILE_M + static_cast<int>(rank) * 128;
                // where this CTA's two boxes of B start: halves of the gate's and the up projection's columns, or
                // 128 consecutive columns
                const int n0 = C::DUAL ? w.nt * C::TILE_N : w.nt * tile_n + static_cast<int>(rank) * 128;
                const int n1 = (C::DUAL && !PAIR) ? n0 : n0 + 64;
                for (int k0 = w.k_begin; k0 < w.k_end; ++k0) {
                    int k = serpentine_k(it, k0, w.k_begin, w.k_end);
                    const int kseg = k >= jb.k_steps0 ? 1 : 0;
                    k -= kseg * jb.k_steps0;
                    if (!(ok = wait_bar_t<true, PAIR>(cx, empty + 8 * r.stage, r.phase ^ 1u, 0x001))) break;
                    if (rank == 0) mbar_arrive_expect_tx(full + 8 * r.stage, PAIR ? 2 * C::STAGE_BYTES : b_bytes + jb.a_rows * 128u);
                    const uint32_t bar = PAIR ? mapa_shared(full + 8 * r.stage, 0) : full + 8 * r.stage;
                    const uint32_t dst = smem_base + r.stage * stage_bytes;
                    const int b0 = C::DUAL ? (PAIR ? static_cast<int>(rank) : 0) : (w.seg | kseg);
                    const int b1 = C::DUAL ? (PAIR ? static_cast<int>(rank) : 1) : (w.seg | kseg);
                    if (PAIR || jb.a_rows == 128) mm_load<PAIR>(dst, ta + kseg, ta + kseg, a_mn, m0, m0 + 64, k * kMmKStep, bar);
                    else mm_tma<PAIR>(dst, ta + kseg, k * kMmKStep, m0, bar);       // the tile's other rows are whatever lies behind: no row of C that exists reads them
                    if constexpr (C::ANY_WIDTH) mm_tma<PAIR>(dst + a_bytes, tb + b0, k * kMmKStep, n0, bar);       // one box of tile_n rows of B^T
                    else mm_load<PAIR>(dst + a_bytes, tb + b0, tb + b1, b_mn, n0, n1, k * kMmKStep, bar);
                    r.advance(stages);
                }
            }
        }
    } else if (warp == 1) {
        // ================================ UMMA issuer =================================
        if (rank == 0 && elect_one()) {
            Ring r;
            bool ok = true;
            int it = 0;
            for (int item; ok && (item = mm_item_at<PAIR>(it)) < p.items; ++it) {
                const MmItem w = mm_item<C::JOBS>(p, item);
                const bool a_mn = p.job[w.job].a_mn, b_mn = p.job[w.job].b_mn;
                const uint32_t idesc = umma_idesc_bf16_f32(PAIR ? 256 : 128, C::ANY_WIDTH ? tile_n : C::BN, a_mn, b_mn);
                const uint32_t a_step = mm_desc_step(a_mn), b_step = mm_desc_step(b_mn);
                const int acc = it & 1, steps = w.k_end - w.k_begin;
                const uint32_t acc_phase = static_cast<uint32_t>(it >> 1) & 1u;
                // the epilogue has drained this accumulator (the tile before the previous one)
                if (!(ok = wait_bar_t<true, PAIR>(cx, acc_empty + 8 * acc, acc_phase ^ 1u, 0x102))) break;
                for (int k = 0; k < steps; ++k) {
                    if (!(ok = wait_bar_t<true, PAIR>(cx, full + 8 * r.stage, r.phase, 0x101))) break;
                    tcgen05_fence_after_sync();
                    const uint32_t as = smem_base + r.stage * stage_bytes;
                    const uint64_t a_desc = mm_desc(as, a_mn), b_desc = mm_desc(as + a_bytes, b_mn);
#pragma unroll
                    for (int kk = 0; kk < kMmKStep / 16; ++kk) {
                        const uint32_t accumulate = (k > 0 || kk > 0) ? 1u : 0u;
                        if constexpr (PAIR)
                            umma_f16_ss_pair(tmem_base + acc * C::BN, a_desc + kk * a_step, b_desc + kk * b_step, idesc, accumulate);
                        else
                            umma_f16_ss(tmem_base + acc * C::BN, a_desc + kk * a_step, b_desc + kk * b_step, idesc, accumulate);
                    }
                    if constexpr (PAIR) umma_commit_pair(empty + 8 * r.stage, 3); else umma_commit(empty + 8 * r.stage);
                    r.advance(stages);
                }
                if (!ok) break;
                if constexpr (PAIR) umma_commit_pair(acc_full + 8 * acc, 3); else umma_commit(acc_full + 8 * acc);
            }
        }
    } else {
        // ================================ epilogue ====================================
        const int e = warp - kMmFirstEpiWarp, q = warp & 3, half = e >> 2;
        BoxWriter<C::BOXES> out(smem_base + C::BOX_OFF + static_cast<uint32_t>(e) * C::BOXES * kEpilogueBoxBytes, box_bar + 8 * e * C::BOX_BARS, lane);
        int it = 0;
        bool ok = true;
        float unit = 1.f;
        if constexpr (EPI == atb::kMmDlogits) unit = mm_unit(p, smem_base + C::BOX_OFF, C::BOXES * kEpilogueBoxBytes, e, lane);
        for (int item; ok && (item = mm_item_at<PAIR>(it)) < p.items; ++it) {
            const MmItem w = mm_item<C::JOBS>(p, item);
            const MmJob& jb = p.job[w.job];
            const int64_t row0 = static_cast<int64_t>(w.mt) * C::TILE_M + rank * 128 + q * 32, col0 = static_cast<int64_t>(w.nt) * tile_n;
            const int acc = it & 1;
            if constexpr (EPI == atb::kMmLinear) {
                // Residual and bias are asked for before the accumulator is waited for: after it, 509 x 2048 x 5464 took 24.1 us instead of 22.0 and
                // 16 x 2048 x 32000 28.4 instead of 26.6.
                const int64_t own0 = col0 + half * C::COLS;
                linear_fetch<C, KEEP32>(tm, p, jb, out, row0, own0);
                const LinearBias<C> bias(p, jb, own0, lane);
                if (!(ok = wait_bar_t<false, PAIR>(cx, acc_full + 8 * acc, static_cast<uint32_t>(it >> 1) & 1u, 0x201))) break;
                tcgen05_fence_after_sync();
                linear_epilogue<C, KEEP32>(tm, p, jb, out, bias, tmem_base + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(acc * C::BN + half * C::COLS), row0,
                                           own0, lane, cx);
            } else {
                if constexpr (EPI == atb::kMmGluBackward)
                    if (row0 < jb.M && col0 + half * C::COLS < jb.N) out.fetch(&tm.c[2], &tm.c[3], col0 + half * C::COLS, row0);
                if (!(ok = wait_bar_t<false, PAIR>(cx, acc_full + 8 * acc, static_cast<uint32_t>(it >> 1) & 1u, 0x201))) break;
                tcgen05_fence_after_sync();
                if (half * C::COLS < tile_n)
                    mm_epilogue<C, EPI, KEEP32>(tm, p, jb, 2 * w.job + w.seg, out, tmem_base + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(acc * C::BN),
                                        half, row0, col0, min(C::COLS, tile_n - half * C::COLS), w.split, unit, lane, cx);
            }
            tcgen05_fence_before_sync();
            __syncwarp();
#ifdef ATB_TEST_WITHHOLD_ACC_ARRIVAL
            // Test build of the timeout path only: the first epilogue warp of CTA 0 keeps back its very first arrival, so the issuer's
            // bounded wait for that accumulator runs out at the CTA's third tile, the CTA aborts, every role returns and
            // atb_device_status reports it.  No UMMA depends on the missing arrival; loads already under way land in their stages.
            if (blockIdx.x == 0 && e == 0 && it == 0) continue;
#endif
            if (lane == 0) {
                if constexpr (PAIR) mbar_arrive_cluster(mapa_shared(acc_empty + 8 * acc, 0));
                else mbar_arrive(acc_empty + 8 * acc);
            }
        }
        if (lane == 0) tma_store_wait_all<0>();
    }

    // ---- teardown: copies in flight land before the shared memory goes; the peer may still arrive here ----
    if (*cx.abort_flag) {
        for (int i = 0; i < 64; ++i) __nanosleep(20000);
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    if constexpr (PAIR) cluster_sync_all();
    if (warp == 1) {
        tcgen05_fence_after_sync();
        if constexpr (PAIR) tmem_dealloc_pair(tmem_base, 2 * C::BN);
        else tmem_dealloc(tmem_base, 2 * C::BN);
    }
}

// ------------------------------------------------------------------------------------------ host
struct MmDevice {
    bool known = false;
    int ordinal = 0, major = 0, minor = 0, sms = 0;
    unsigned int* flag = nullptr;
};
MmDevice g_mm_devices[64];
std::mutex g_mm_mutex;

bool operand_map(CUtensorMap* m, const atb::MmOperand& o, bool mn_major, int64_t mn, int64_t K, int rows = 64) {
    return make_map_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, o.base, static_cast<uint64_t>(mn_major ? mn : K),
                       static_cast<uint64_t>(mn_major ? K : mn), static_cast<uint64_t>(o.ld) * 2, 64, static_cast<uint32_t>(rows), CU_TENSOR_MAP_SWIZZLE_128B);
}

// Eight values from element `at` on, FP32 or bf16 in memory.
template <bool F32>
__device__ __forceinline__ void load8(const void* src, int64_t at, float (&v)[8]) {
    if constexpr (F32) {
        const float4* const s = reinterpret_cast<const float4*>(static_cast<const float*>(src) + at);
        const float4 a = s[0], b = s[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(src) + at);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 f = unpack_bf16(w[e]);
            v[2 * e] = f.x; v[2 * e + 1] = f.y;
        }
    }
}
template <bool F32>
__device__ __forceinline__ void store8(void* dst, int64_t at, const float (&v)[8]) {
    if constexpr (F32) {
        float4* const d = reinterpret_cast<float4*>(static_cast<float*>(dst) + at);
        d[0] = make_float4(v[0], v[1], v[2], v[3]);
        d[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(dst) + at) =
            make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
}

// Joins the K ranges of split products: sums of the ranges in their order, then what the epilogue would have done.
// src: [splits][split_rows][cols]; eight columns per thread.
template <int EPI, bool KEEP32>
__global__ void __launch_bounds__(256) bf16_mm_join_kernel(const __grid_constant__ MmJoin p) {
    grid_dependency_wait();
    grid_dependency_launch();
    const auto put = [](void* C, int64_t at, const uint32_t (&o)[4]) {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(C) + at) = make_uint4(o[0], o[1], o[2], o[3]);
    };
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < p.all; i += static_cast<int64_t>(gridDim.x) * 256) {
        int j = 0;
        if constexpr (EPI == kMmPlain)
            while (j + 1 < p.n_jobs && i >= p.job[j + 1].first) ++j;
        const MmJoinJob& q = p.job[j];
        const auto sum = [&](int64_t m, int64_t col, float (&v)[8]) {
            const float* src = q.src + m * q.cols + col;
            float4 a = *reinterpret_cast<const float4*>(src), b = *reinterpret_cast<const float4*>(src + 4);
            for (int s = 1; s < q.splits; ++s) {
                src += q.split_rows * q.cols;
                const float4 c = *reinterpret_cast<const float4*>(src), d = *reinterpret_cast<const float4*>(src + 4);
                a.x += c.x; a.y += c.y; a.z += c.z; a.w += c.w;
                b.x += d.x; b.y += d.y; b.z += d.z; b.w += d.w;
            }
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        };
        const int64_t per_row = q.N / 8, at = i - q.first;
        const int64_t m = at / (per_row * q.n_segs), g8 = at - m * per_row * q.n_segs;
        const int seg = g8 >= per_row ? 1 : 0;
        const int64_t n = (g8 - seg * per_row) * 8;
        float v[8];
        sum(m, seg * q.N + n, v);
        uint32_t o[4];
        if constexpr (EPI == kMmPlain) {
            const float factor = q.factor ? *q.factor : 1.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= factor;
            if (q.C32) {
                float* dst = q.C32 + m * q.N + n;
#pragma unroll
                for (int e = 0; e < 8; ++e) dst[e] = q.add ? dst[e] + v[e] : v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                put(q.C[seg], m * q.ldc[seg] + n, o);
            }
        } else if constexpr (EPI == atb::kMmLinear) {
            float b[8], r[8] = {};
            load_bias(p.bias, p.bias32, n, q.N, b);
            if (p.R) load8<KEEP32>(p.R, m * p.ldr + n, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += b[e];
            if (q.C[1]) {
                if (p.z32) store8<true>(q.C[1], m * q.ldc[1] + n, v);
                else store8<false>(q.C[1], m * q.ldc[1] + n, v);
            }
            with_linear_act(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 a = act_value<act.value>(make_float2(v[2 * e], v[2 * e + 1]));
                    v[2 * e] = a.x + r[2 * e];
                    v[2 * e + 1] = a.y + r[2 * e + 1];
                }
            });
            store8<KEEP32>(q.C[0], m * q.ldc[0] + n, v);
        } else if constexpr (EPI == atb::kMmGlu) {
            float u[8];
            sum(m, q.N + n, u);
            with_act(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = glu_pair<act.value>(make_float2(v[2 * e], v[2 * e + 1]), make_float2(u[2 * e], u[2 * e + 1]));
            });
            put(q.C[0], m * q.ldc[0] + n, o);
            if constexpr (KEEP32) {
                const auto put32 = [&](void* C, int64_t ld, const float (&f)[8]) {
                    float4* const dst = reinterpret_cast<float4*>(static_cast<float*>(C) + m * ld + n);
                    dst[0] = make_float4(f[0], f[1], f[2], f[3]);
                    dst[1] = make_float4(f[4], f[5], f[6], f[7]);
                };
                put32(q.C[1], q.ldc[1], v);
                put32(q.C[2], q.ldc[2], u);
            } else if (q.C[1]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                put(q.C[1], m * q.ldc[1] + n, o);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = pack_bf16(u[2 * e], u[2 * e + 1]);
                put(q.C[2], m * q.ldc[2] + n, o);
            }
        } else {
            float2 g[4], u[4];
            const auto load = [&](const void* src, float2 (&f)[4]) {
                if constexpr (KEEP32) {
                    const float4* const at4 = reinterpret_cast<const float4*>(static_cast<const float*>(src) + m * q.N + n);
                    const float4 a = at4[0], b = at4[1];
                    f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w);
                    f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
                } else {
                    const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(src) + m * q.N + n);
                    f[0] = unpack_bf16(a.x); f[1] = unpack_bf16(a.y); f[2] = unpack_bf16(a.z); f[3] = unpack_bf16(a.w);
                }
            };
            load(p.G, g);
            load(p.U, u);
            uint32_t o2[4];
            with_act(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) glu_backward_pair<act.value>(g[e], u[e], make_float2(v[2 * e], v[2 * e + 1]), o[e], o2[e]);
            });
            put(q.C[0], m * q.ldc[0] + n, o);
            put(q.C[1], m * q.ldc[1] + n, o2);
        }
    }
}

// A is stored along K and has so few rows that one box holds them.
bool few_rows(const atb::MmProblem& q) { return q.layout != atb::kMmTN && q.M <= 64; }

// How a launch is laid out on the SMs: the form, the K ranges of each product, and the order of the products in the list of
// work items (longest items first).
struct MmPlan {
    bool pair = false, split = false;
    int width = 128;                       // columns of a tile of a single CTA (kMmRowStats, kMmDlogits)
    int splits[kMmGroup] = {1, 1, 1}, order[kMmGroup] = {0, 1, 2};
};

bool can_split(int epilogue) { return epilogue != atb::kMmRowStats && epilogue != atb::kMmDlogits; }
int64_t accumulator_columns(const atb::MmProblem& q) { return q.N * (q.epilogue == atb::kMmGlu ? 2 : q.n_segs); }
size_t partial_bytes(const atb::MmProblem& q, int splits) {
    return splits > 1 ? static_cast<size_t>(splits) * static_cast<size_t>(atb::round_up(q.M, 32)) * static_cast<size_t>(accumulator_columns(q)) * sizeof(float) : 0;
}

// Steps that the slowest unit has: items in order of their length, dealt out to and fro (mm_item_at).  Three units are looked
// at; where there are many rounds, all are close to the even share, unless one of the longest items is more than that.
double slowest_unit(const int64_t* count, const double* length, int n, int units) {
    int64_t items = 0;
    double work = 0, shortest = length[n - 1];
    for (int j = 0; j < n; ++j) {
        items += count[j];
        work += static_cast<double>(count[j]) * length[j];
    }
    const int64_t rounds = atb::ceil_div(items, units);
    if (rounds > 8) return std::max(work / units + 0.5 * shortest, length[0] + static_cast<double>(rounds - 1) * shortest);
    double most = 0;
    for (const int u : {0, units / 2, units - 1}) {
        double load = 0;
        for (int64_t r = 0; r < rounds; ++r) {
            int64_t at = r * units + ((r & 1) ? units - 1 - u : u);
            if (at >= items) continue;
            int j = 0;
            while (at >= count[j]) at -= count[j++];
            load += length[j];
        }
        if (load > most) most = load;
    }
    return most;
}

// Cycles of the candidates, by what measured: a K-step of 64 takes 512 cycles in both forms (the pair's 256 x 256 tile is
// bound by the tensor cores; the single CTA's 128 x 128 tile has half the reuse, and its 32 KB per step arrive no
// faster), 650 where A is a few rows and B alone has to arrive, from memory; all operands come from memory at 3400 bytes per
// cycle, if that is more; the last work item 2500 more to fill and drain, and joining K ranges 4000 for a launch and the FP32
// sums, written and read once, at 3 KB per cycle.
MmPlan make_plan(const atb::MmProblem* q, int n) {
    MmPlan best;
    double least = 1e300;
    int64_t k_steps[kMmGroup], longest = 1;
    double operand_bytes = 0;
    bool few = true;
    for (int j = 0; j < n; ++j) {
        few = few && few_rows(q[j]);
        operand_bytes += 2.0 * static_cast<double>(q[j].K * q[j].k_segs) * static_cast<double>(q[j].M + accumulator_columns(q[j]));
        k_steps[j] = atb::ceil_div(q[j].K, kMmKStep) * q[j].k_segs;
        if (k_steps[j] > longest) longest = k_steps[j];
    }
    for (int form = 0; form < 2; ++form) {
        const int tile = form ? 256 : 128, units = form ? atb::kSmCount / 2 : atb::kSmCount;
        int64_t tiles[kMmGroup], longest_tiles = 0;        // longest_tiles: of the products with the longest K
        bool tall = false;                             // a pair needs more than one CTA's rows somewhere
        for (int j = 0; j < n; ++j) {
            tall = tall || q[j].M > 128;
            tiles[j] = atb::ceil_div(q[j].M, tile) * atb::ceil_div(accumulator_columns(q[j]), tile);
            if (k_steps[j] == longest) longest_tiles += tiles[j];
        }
        if (form && !tall) continue;
        const double step = few && !form ? 650.0 : 512.0;
        for (const int s : {1, 2, 3, 4, 6, 8, 12, 16}) {
            if (s > 1 && longest_tiles * s > 4ll * units) break;
            MmPlan c;
            c.pair = form == 1;
            double bytes = 0, len[kMmGroup];
            for (int j = 0; j < n; ++j) {
                // ranges of about the length that s ranges of the longest K have, at least 4 steps each
                int64_t r = (k_steps[j] * s + longest / 2) / longest;
                if (r > k_steps[j] / 4) r = k_steps[j] / 4;
                if (r < 1 || !can_split(q[j].epilogue)) r = 1;
                c.splits[j] = static_cast<int>(r);
                len[j] = static_cast<double>(k_steps[j]) / static_cast<double>(r);
                if (r > 1) { c.split = true; bytes += 2.0 * static_cast<double>(partial_bytes(q[j], c.splits[j])); }
            }
            if (s > 1 && !c.split) break;
            for (int i = 1; i < n; ++i)                // longest items first
                for (int k = i; k > 0 && len[c.order[k]] > len[c.order[k - 1]]; --k) std::swap(c.order[k], c.order[k - 1]);
            int64_t count[kMmGroup];
            double length[kMmGroup];
            for (int i = 0; i < n; ++i) { count[i] = tiles[c.order[i]] * c.splits[c.order[i]]; length[i] = len[c.order[i]]; }
            const double t = std::max(step * slowest_unit(count, length, n, units), operand_bytes / 3400.0) + 2500.0 +
                             (c.split ? 4000.0 + bytes / 3000.0 : 0.0);
            if (t < least * 0.98) { least = t; best = c; }
        }
    }
    if (!best.pair && !can_split(q->epilogue) && few) {
        // A few rows' head reads W once, and an SM draws no more than its share of the memory's rate: the width (multiples of 16) that
        // leaves the slowest SM the fewest columns, each tile counting 24 more.  V = 20731, D = 2160: 80 instead of 128 columns,
        // two rounds each.
        int64_t fewest = INT64_MAX;
        for (int width = 128; width >= 16; width -= 16) {
            const int64_t columns = atb::ceil_div(atb::ceil_div(q->N, width), atb::kSmCount) * (width + 24);
            if (columns < fewest) { fewest = columns; best.width = width; }
        }
    }
    return best;
}

// Output boxes of 32 rows x 128 bytes.
template <class T>
bool output_map(CUtensorMap* m, const void* base, int64_t N, int64_t M, int64_t ld) {
    constexpr bool F32 = sizeof(T) == 4;
    return make_map_2d(m, F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, sizeof(T), base, static_cast<uint64_t>(N),
                       static_cast<uint64_t>(M), static_cast<uint64_t>(ld) * sizeof(T), 128 / sizeof(T), 32, CU_TENSOR_MAP_SWIZZLE_128B);
}

// One kernel over the n products of q.  EPI == kMmPlain: bf16, FP32, or the sums of K ranges in `partial`.
template <bool PAIR, int EPI, bool KEEP32 = false>
atb_status_t launch(const atb::MmProblem* q, int n, const MmPlan& plan, char* partial, const MmDevice& dev, cudaStream_t stream) {
    using C = MmCfg<PAIR, EPI>;
    MmMaps<C::JOBS> tm;
    MmParams p = {};
    size_t offset[kMmGroup], end = 0;
    for (int j = 0; j < n; ++j) { offset[j] = end; end += partial_bytes(q[j], plan.splits[j]); }
    int64_t items = 0;
    for (int i = 0; i < C::JOBS; ++i) {
        if (i >= n) {                      // maps that are not used are copies of the first product's
            tm.a[2 * i] = tm.a[2 * i + 1] = tm.a[0];
            tm.b[2 * i] = tm.b[2 * i + 1] = tm.b[0];
            tm.c[2 * i] = tm.c[2 * i + 1] = tm.c[0];
            continue;
        }
        const int j = plan.order[i];
        const atb::MmProblem& x = q[j];
        const bool a_mn = x.layout == atb::kMmTN, b_mn = x.layout != atb::kMmNT;
        const int n_segs = C::DUAL ? 1 : (x.epilogue == atb::kMmGlu ? 2 : x.n_segs);     // a split gated product: two side by side
        const int n_b = C::DUAL || n_segs == 2 ? 2 : x.k_segs;
        const bool few = !PAIR && few_rows(x);                     // one box of A holds every row
        const int a_box = few ? static_cast<int>(atb::round_up(x.M, 8)) : 64;
        for (int s = 0; s < 2; ++s) {
            if (s >= x.k_segs) tm.a[2 * i + s] = tm.a[2 * i];
            else if (!operand_map(&tm.a[2 * i + s], x.A[s], a_mn, x.M, x.K, a_box)) return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for A");
            if (s >= n_b) tm.b[2 * i + s] = tm.b[2 * i];
            else if (!operand_map(&tm.b[2 * i + s], x.B[s], b_mn, x.N, x.K, C::ANY_WIDTH ? plan.width : 64)) return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for B");
        }
        MmJob& jb = p.job[i];
        jb.M = x.M; jb.N = x.N;
        jb.a_mn = a_mn; jb.b_mn = b_mn;
        jb.a_rows = few ? a_box : 128;
        jb.m_tiles = static_cast<int>(atb::ceil_div(x.M, C::TILE_M));
        jb.n_tiles = static_cast<int>(atb::ceil_div(x.N, C::ANY_WIDTH ? plan.width : C::TILE_N));
        jb.n_segs = n_segs;
        jb.k_steps0 = static_cast<int>(atb::ceil_div(x.K, kMmKStep));
        jb.k_steps = jb.k_steps0 * x.k_segs;
        jb.splits = EPI == kMmPlain ? plan.splits[j] : 1;
        jb.first_item = static_cast<int>(items);
        items += static_cast<int64_t>(jb.m_tiles) * jb.n_tiles * jb.n_segs * jb.splits;
        if (items > (1ll << 30)) return atb::fail(ATB_ERR_BAD_SHAPE, "too many output tiles");
        if constexpr (EPI == kMmPlain) {
            jb.fp32 = jb.splits > 1 || x.epilogue == atb::kMmAccumulate;
            jb.split_rows = jb.splits > 1 ? atb::round_up(x.M, 32) : 0;
            jb.add = jb.splits == 1 && jb.fp32 && !x.first;
            jb.factor = jb.splits == 1 ? x.factor : nullptr;
            for (int s = 0; s < 2; ++s) {
                CUtensorMap* const m = &tm.c[2 * i + s];
                bool ok = true;
                if (s >= n_segs) *m = tm.c[2 * i];
                else if (jb.splits > 1)     // a map per segment, so that each clips at its own last column
                    ok = output_map<float>(m, reinterpret_cast<float*>(partial + offset[j]) + s * x.N, x.N, jb.splits * jb.split_rows, x.N * n_segs);
                else if (jb.fp32) ok = output_map<float>(m, x.C32, x.N, x.M, x.N);
                else ok = output_map<__nv_bfloat16>(m, x.C[s], x.N, x.M, x.ldc[s]);
                if (!ok) return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for C");
            }
        } else if constexpr (EPI == atb::kMmLinear) {
            const auto map = [&](int s, const void* base, int64_t ld, bool fp32) {
                if (!base) { tm.c[s] = tm.c[0]; return true; }                         // not used: any valid map
                return fp32 ? output_map<float>(&tm.c[s], base, x.N, x.M, ld) : output_map<__nv_bfloat16>(&tm.c[s], base, x.N, x.M, ld);
            };
            if (!map(0, x.C[0], x.ldc[0], KEEP32) || !map(1, x.C[1], x.ldc[1], x.z32) || !map(2, x.R, x.ldr, KEEP32))
                return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for C");
            tm.c[3] = tm.c[0];
            p.bias = x.bias; p.bias32 = x.bias32; p.residual = x.R != nullptr;
            p.kept = !x.C[1] ? 0 : x.z32 ? kKeptF32 : kKeptBf16;
        } else {
            const void* const c[4] = {x.C[0], x.C[1], EPI == atb::kMmGluBackward ? x.G : x.C[2], EPI == atb::kMmGluBackward ? x.U : nullptr};
            for (int s = 0; s < 4; ++s) {
                if (!c[s]) { tm.c[s] = s ? tm.c[0] : tm.a[0]; continue; }              // not written: any valid map
                const int64_t ld = EPI == atb::kMmGluBackward && s >= 2 ? x.N : x.ldc[s];
                const bool fp32 = KEEP32 && (EPI == atb::kMmGlu ? s == 1 || s == 2 : s >= 2);        // g and u
                if (!(fp32 ? output_map<float>(&tm.c[s], c[s], x.N, x.M, ld) : output_map<__nv_bfloat16>(&tm.c[s], c[s], x.N, x.M, ld)))
                    return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for C");
            }
        }
    }
    int a_rows = 0;
    for (int i = 0; i < n; ++i) a_rows = std::max(a_rows, p.job[i].a_rows);
    p.a_bytes = static_cast<uint32_t>(a_rows) * 128u;          // a_rows is a multiple of 8: whole swizzle atoms of 1 KB
    p.tile_n = C::ANY_WIDTH ? plan.width : C::TILE_N;
    p.b_bytes = C::ANY_WIDTH ? static_cast<uint32_t>(plan.width) * 128u : kMmTileBytes;
    p.stages = std::min<int>(C::MOST_STAGES, C::BOX_OFF / (p.a_bytes + p.b_bytes));
    p.dl = q->C[0]; p.dl_ld = q->ldc[0];
    p.n_jobs = n;
    p.items = static_cast<int>(items);
    p.error_flag = dev.flag;
    p.act = q->act; p.save = q->C[1] != nullptr;
    p.labels = q->labels; p.ignore_index = q->ignore_index; p.col0 = q->col0;
    p.stats = q->stats; p.stats_ld = q->stats_ld; p.label_logit = q->label_logit;
    p.lse = q->lse; p.scale = q->scale;
    p.unit = q->unit; p.rows = q->M; p.first = q->first;
    const int units = PAIR ? dev.sms / 2 : dev.sms;
    const int n_units = static_cast<int>(items < units ? items : units);
    auto kernel = bf16_mm_kernel<PAIR, EPI, KEEP32>;
    cudaError_t e = cudaSuccess;
    static std::atomic<uint64_t> allowed{0};         // devices on which this kernel has its shared memory allowed
    const uint64_t bit = 1ull << dev.ordinal;
    if (!(allowed.load(std::memory_order_acquire) & bit)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(C::SMEM_BYTES));
        if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
        allowed.fetch_or(bit, std::memory_order_release);
    }
    e = atb::launch_dependent(kernel, static_cast<unsigned>(PAIR ? 2 * n_units : n_units), kMmThreads, PAIR ? 2u : 1u, C::SMEM_BYTES, stream, tm, p);
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "bf16 product launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

template <int EPI, bool KEEP32>
atb_status_t join(const atb::MmProblem* q, int n, const MmPlan& plan, const char* partial, const MmDevice& dev, cudaStream_t stream) {
    MmJoin p = {};
    size_t offset = 0;
    for (int j = 0; j < n; ++j) {
        if (plan.splits[j] > 1) {
            MmJoinJob& jb = p.job[p.n_jobs++];
            jb.M = q[j].M; jb.N = q[j].N;
            jb.n_segs = EPI == atb::kMmGlu ? 1 : q[j].n_segs;
            jb.cols = accumulator_columns(q[j]);
            jb.src = reinterpret_cast<const float*>(partial + offset);
            jb.splits = plan.splits[j];
            jb.split_rows = atb::round_up(q[j].M, 32);
            for (int i = 0; i < 3; ++i) { jb.C[i] = q[j].C[i]; jb.ldc[i] = q[j].ldc[i]; }
            jb.C32 = q[j].epilogue == atb::kMmAccumulate ? q[j].C32 : nullptr;
            jb.add = !q[j].first;
            jb.factor = q[j].factor;
            jb.first = p.all;
            p.all += jb.M * (jb.N / 8) * jb.n_segs;
        }
        offset += partial_bytes(q[j], plan.splits[j]);
    }
    p.act = q->act;
    p.G = q->G; p.U = q->U;
    p.bias = q->bias; p.bias32 = q->bias32; p.R = q->R; p.ldr = q->ldr; p.z32 = q->z32;
    const int64_t blocks = atb::ceil_div(p.all, 256), most = static_cast<int64_t>(dev.sms) * 8;
    const cudaError_t e = atb::launch_dependent(bf16_mm_join_kernel<EPI, KEEP32>, static_cast<unsigned>(blocks < most ? blocks : most), 256u, 1u, 0, stream, p);
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "bf16 product join launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

template <int EPI, bool KEEP32 = false>
atb_status_t run(const atb::MmProblem* q, int n, const MmPlan& plan, char* partial, const MmDevice& dev, cudaStream_t stream) {
    if (!plan.split) return plan.pair ? launch<true, EPI, KEEP32>(q, n, plan, partial, dev, stream) : launch<false, EPI, KEEP32>(q, n, plan, partial, dev, stream);
    if constexpr (EPI == atb::kMmRowStats || EPI == atb::kMmDlogits) {
        return atb::fail(ATB_ERR_BAD_ARGUMENT, "this epilogue takes whole sums");
    } else {
        if (!partial) return atb::fail(ATB_ERR_NULL_POINTER, "a product that is split along K needs room for its sums");
        const atb_status_t s = plan.pair ? launch<true, kMmPlain>(q, n, plan, partial, dev, stream) : launch<false, kMmPlain>(q, n, plan, partial, dev, stream);
        return s != ATB_OK ? s : join<EPI, KEEP32>(q, n, plan, partial, dev, stream);
    }
}

}  // namespace

namespace atb {

static atb_status_t mm_device(const MmDevice** out) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return fail(ATB_ERR_CUDA, "cudaGetDevice: %s", cudaGetErrorString(e));
    if (dev < 0 || dev >= 64) return fail(ATB_ERR_UNSUPPORTED_DEVICE, "device ordinal %d out of range", dev);
    std::lock_guard<std::mutex> lock(g_mm_mutex);
    MmDevice& d = g_mm_devices[dev];
    if (!d.known) {
        d.ordinal = dev;
        cudaDeviceGetAttribute(&d.major, cudaDevAttrComputeCapabilityMajor, dev);
        cudaDeviceGetAttribute(&d.minor, cudaDevAttrComputeCapabilityMinor, dev);
        cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev);
        if (d.major == 10 && d.minor == 0) {
            e = cudaGetSymbolAddress(reinterpret_cast<void**>(&d.flag), g_mm_error_flag);
            if (e != cudaSuccess) return fail(ATB_ERR_CUDA, "cudaGetSymbolAddress: %s", cudaGetErrorString(e));
        }
        d.known = true;
    }
    if (d.major != 10 || d.minor != 0)
        return fail(ATB_ERR_UNSUPPORTED_DEVICE, "compute capability %d.%d; this library runs on 10.0 only", d.major, d.minor);
    *out = &d;
    return ATB_OK;
}

atb_status_t op_device(int* num_sms) {
    const MmDevice* d = nullptr;
    const atb_status_t s = mm_device(&d);
    if (s == ATB_OK) *num_sms = d->sms;
    return s;
}

unsigned int take_mm_error_flag() {
    unsigned int flag = 0;
    if (cudaMemcpyFromSymbol(&flag, g_mm_error_flag, sizeof flag) != cudaSuccess) return 0;
    if (flag != 0) {
        const unsigned int zero = 0;
        cudaMemcpyToSymbol(g_mm_error_flag, &zero, sizeof zero);
    }
    return flag;
}

int64_t mm_stats_per_row(int64_t M, int64_t N, int64_t K) {
    const MmProblem q = mm_sizes(kMmNT, kMmRowStats, M, N, K);
    const MmPlan plan = make_plan(&q, 1);
    // two groups of columns per tile, or one of at most 64; the last tile may end in its first
    const int tile = plan.pair ? 256 : plan.width, group = plan.pair ? 128 : 64, groups = tile > group ? 2 : 1;
    const int64_t whole = (N - 1) / tile, rest = N - whole * tile;
    return whole * groups + (rest > group ? 2 : 1);
}

size_t mm_partial_bytes(const MmProblem* q, int n) {
    const MmPlan plan = make_plan(q, n);
    size_t bytes = 0;
    for (int j = 0; j < n; ++j) bytes += partial_bytes(q[j], plan.splits[j]);
    return bytes;
}

atb_status_t mm_launch(const MmProblem* q, int n, void* partial, cudaStream_t stream) {
    const MmDevice* dev = nullptr;
    const atb_status_t s = mm_device(&dev);
    if (s != ATB_OK) return s;
    const MmPlan plan = make_plan(q, n);
    char* const room = static_cast<char*>(partial);
    switch (q->epilogue) {
        case kMmStore: case kMmAccumulate: return run<kMmPlain>(q, n, plan, room, *dev, stream);
        case kMmGlu: return q->keep32 ? run<kMmGlu, true>(q, n, plan, room, *dev, stream) : run<kMmGlu>(q, n, plan, room, *dev, stream);
        case kMmGluBackward: return q->keep32 ? run<kMmGluBackward, true>(q, n, plan, room, *dev, stream) : run<kMmGluBackward>(q, n, plan, room, *dev, stream);
        case kMmRowStats: return run<kMmRowStats>(q, n, plan, room, *dev, stream);
        case kMmDlogits: return run<kMmDlogits>(q, n, plan, room, *dev, stream);
        case kMmLinear: return q->y32 ? run<kMmLinear, true>(q, n, plan, room, *dev, stream) : run<kMmLinear>(q, n, plan, room, *dev, stream);
    }
    return fail(ATB_ERR_BAD_ARGUMENT, "no product kernel for epilogue %d", static_cast<int>(q->epilogue));
}

}  // namespace atb
