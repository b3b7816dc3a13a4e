// BF16 x BF16 products with FP32 accumulation for the gated feed-forward block and the linear cross entropy (sm_100a).
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
//   single  128 x 128 tile: four times as many tiles for outputs that would leave most of the SMs idle
// Every wait is bounded (see atb_gemm_device.cuh).
#include <atomic>
#include <type_traits>

#include "atb_bf16_mm.h"
#include "atb_gemm_device.cuh"
#include "glu.cuh"

namespace {

using namespace glu;

__device__ unsigned int g_mm_error_flag = 0;

constexpr int kMmKStep = 64;
constexpr uint32_t kMmBoxBytes = 64 * 128;              // 64 rows of 64 bf16
constexpr uint32_t kMmTileBytes = 2 * kMmBoxBytes;      // a CTA's part of A, or of B, for one K-step
constexpr int kMmEpiWarps = 8, kMmFirstEpiWarp = 2;
constexpr int kMmThreads = (kMmFirstEpiWarp + kMmEpiWarps) * 32;

struct MmMaps {
    CUtensorMap a[2], b[2], c[3];
};

struct MmParams {
    int64_t M, N;
    int m_tiles, n_tiles, n_segs;      // n_tiles: of one segment
    int k_steps0, k_steps;             // steps of the first K segment, of both
    unsigned int* error_flag;
    int splits;                        // the K loop is cut into this many ranges, units of work of their own
    int64_t split_rows;                // kMmAccumulate: rows of the output between the sums of one range and the next
    int add;                           // kMmAccumulate: added to the output
    int act, save;
    const __nv_bfloat16 *G, *U;
    const int64_t* labels;
    int64_t ignore_index, col0;
    float2* stats;
    int64_t stats_ld;
    float* label_logit;
    const float *lse, *scale;
};

struct MmJoin {
    int64_t M, N, cols, split_rows;
    int n_segs, splits, act, add;
    const float* src;
    void* C[3];
    int64_t ldc[3];
    float* C32;
    const __nv_bfloat16 *G, *U;
};

template <bool PAIR, int EPI>
struct MmCfg {
    static constexpr int BN = PAIR ? 256 : 128;             // accumulator columns
    static constexpr int TILE_M = PAIR ? 256 : 128;
    static constexpr bool DUAL = EPI == atb::kMmGlu;        // half of the columns from B[0], half from B[1]
    static constexpr int TILE_N = DUAL ? BN / 2 : BN;       // columns of C per tile
    static constexpr int COLS = DUAL ? 64 : BN / 2;         // columns of C of an epilogue warp (a 64-column tile has one group)
    static constexpr int BOXES = (EPI == atb::kMmGlu || EPI == atb::kMmGluBackward) ? 2 : 1;   // staging boxes of a warp
    static constexpr int STAGES = BOXES == 2 ? 5 : 6;
    static constexpr uint32_t STAGE_BYTES = 2 * kMmTileBytes;
    static constexpr uint32_t BOX_OFF = STAGES * STAGE_BYTES;
    static constexpr uint32_t BAR_OFF = BOX_OFF + kMmEpiWarps * BOXES * kEpilogueBoxBytes;
    static constexpr uint32_t SMEM_BYTES = 1024 + BAR_OFF + 8 * (2 * STAGES + 4) + 16;
    static_assert(SMEM_BYTES <= kSmemBudget, "shared memory");
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 b2 = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b2);
}

// dg = dh u act'(g) and du = dh act(g) of two neighbours, g and u packed bf16.
template <int ACT>
__device__ __forceinline__ void glu_backward_pair(uint32_t gw, uint32_t uw, float dh0, float dh1, uint32_t& dg, uint32_t& du) {
    float a0, s0, a1, s1;
    act_value_slope<ACT>(__uint_as_float(gw << 16), a0, s0);
    act_value_slope<ACT>(__uint_as_float(gw & 0xFFFF0000u), a1, s1);
    dg = pack_bf16(dh0 * __uint_as_float(uw << 16) * s0, dh1 * __uint_as_float(uw & 0xFFFF0000u) * s1);
    du = pack_bf16(dh0 * a0, dh1 * a1);
}

// A warp's staging boxes of 32 rows x 64 bf16 or 32 fp32 (128-byte swizzle), used in turn; each leaves by a TMA store, or is
// added to memory by one, which clips at the edges of the output.
template <int BOXES>
struct BoxWriter {
    uint32_t base;
    int lane, next = 0;
    __device__ BoxWriter(uint32_t b, int l) : base(b), lane(l) {}
    __device__ __forceinline__ void put(const CUtensorMap* map, const uint32_t (&o)[32], int64_t col, int64_t row0, bool inside, bool add = false) {
        if (lane == 0) tma_store_wait_read<BOXES - 1>();       // the store that last used this box has read it
        __syncwarp();
        const uint32_t box = base + next * kEpilogueBoxBytes, row = box + lane * 128, sw = lane & 7;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(row + ((static_cast<uint32_t>(j) ^ sw) << 4)),
                         "r"(o[4 * j]), "r"(o[4 * j + 1]), "r"(o[4 * j + 2]), "r"(o[4 * j + 3]) : "memory");
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            if (inside) {
                if (add) tma_reduce_add_2d(map, box, static_cast<int>(col), static_cast<int>(row0));
                else tma_store_2d(map, box, static_cast<int>(col), static_cast<int>(row0));
            }
            tma_store_commit();                                // an empty group keeps the count of groups per box
        }
        next = next + 1 == BOXES ? 0 : next + 1;
    }
};

// ------------------------------------------------------------------------------------------ epilogue of one warp
// Rows row0 .. row0 + 31 (one per lane); t_addr: the warp's lanes of the tile's accumulator, column 0; half: which of
// the tile's column groups this warp has; col0: first column of the tile in C.
template <class C, int EPI>
__device__ __forceinline__ void mm_epilogue(const MmMaps& tm, const MmParams& p, BoxWriter<C::BOXES>& out, uint32_t t_addr, int half,
                                            int64_t row0, int64_t col0, int seg, int split, int lane) {
    const int64_t row = row0 + lane;
    const bool row_in = row < p.M, warp_in = row0 < p.M;
    col0 += half * C::COLS;
    t_addr += half * C::COLS;
    if constexpr (EPI == atb::kMmStore) {
#pragma unroll 1
        for (int c = 0; c < C::COLS; c += 64) {
            uint32_t v[32], w[32], o[32];
            tmem_ld_32x32b_x32(t_addr + c, v);
            tmem_ld_32x32b_x32(t_addr + c + 32, w);
            tmem_ld_wait_for(v);
            tmem_ld_wait_for(w);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                o[e] = pack_bf16(__uint_as_float(v[2 * e]), __uint_as_float(v[2 * e + 1]));
                o[16 + e] = pack_bf16(__uint_as_float(w[2 * e]), __uint_as_float(w[2 * e + 1]));
            }
            out.put(&tm.c[seg], o, col0 + c, row0, warp_in && col0 + c < p.N);
        }
    } else if constexpr (EPI == atb::kMmAccumulate) {
        // FP32: rows of this K range's sums (see MmParams::split_rows), or added to what is there
#pragma unroll 1
        for (int c = 0; c < C::COLS; c += 32) {
            uint32_t v[32];
            tmem_ld_32x32b_x32(t_addr + c, v);
            tmem_ld_wait_for(v);
            out.put(&tm.c[seg], v, col0 + c, split * p.split_rows + row0, warp_in && col0 + c < p.N, p.add);
        }
    } else if constexpr (EPI == atb::kMmGlu) {
        // accumulator columns 0 .. TILE_N - 1 hold g, the next TILE_N hold u
        with_act(p.act, [&](auto act) {
            uint32_t h[32], og[32], ou[32];
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                uint32_t g[32], u[32];
                tmem_ld_32x32b_x32(t_addr + 32 * part, g);
                tmem_ld_32x32b_x32(t_addr + C::TILE_N + 32 * part, u);
                tmem_ld_wait_for(g);
                tmem_ld_wait_for(u);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float a0, a1, slope;
                    act_value_slope<act.value>(__uint_as_float(g[2 * e]), a0, slope);
                    act_value_slope<act.value>(__uint_as_float(g[2 * e + 1]), a1, slope);
                    h[16 * part + e] = pack_bf16(a0 * __uint_as_float(u[2 * e]), a1 * __uint_as_float(u[2 * e + 1]));
                    og[16 * part + e] = pack_bf16(__uint_as_float(g[2 * e]), __uint_as_float(g[2 * e + 1]));
                    ou[16 * part + e] = pack_bf16(__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1]));
                }
            }
            const bool inside = warp_in && col0 < p.N;
            out.put(&tm.c[0], h, col0, row0, inside);
            if (p.save) {
                out.put(&tm.c[1], og, col0, row0, inside);
                out.put(&tm.c[2], ou, col0, row0, inside);
            }
        });
    } else if constexpr (EPI == atb::kMmGluBackward) {
        with_act(p.act, [&](auto act) {
#pragma unroll 1
            for (int c = 0; c < C::COLS; c += 64) {
                uint32_t og[32], ou[32];
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const int64_t col = col0 + c + 32 * part;
                    uint32_t dh[32];
                    tmem_ld_32x32b_x32(t_addr + c + 32 * part, dh);
                    uint4 g[4], u[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        g[j] = u[j] = make_uint4(0, 0, 0, 0);
                        if (row_in && col + 8 * j < p.N) {         // N is a multiple of 8
                            g[j] = *reinterpret_cast<const uint4*>(p.G + row * p.N + col + 8 * j);
                            u[j] = *reinterpret_cast<const uint4*>(p.U + row * p.N + col + 8 * j);
                        }
                    }
                    tmem_ld_wait_for(dh);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint32_t gw = reinterpret_cast<const uint32_t*>(g)[e], uw = reinterpret_cast<const uint32_t*>(u)[e];
                        glu_backward_pair<act.value>(gw, uw, __uint_as_float(dh[2 * e]), __uint_as_float(dh[2 * e + 1]), og[16 * part + e],
                                                     ou[16 * part + e]);
                    }
                }
                const bool inside = warp_in && col0 + c < p.N;
                out.put(&tm.c[0], og, col0 + c, row0, inside);
                out.put(&tm.c[1], ou, col0 + c, row0, inside);
            }
        });
    } else if constexpr (EPI == atb::kMmRowStats) {
        // the label's column, counted from this warp's first one
        int64_t label = -1;
        if (row_in) label = p.labels[row] - p.col0 - col0;
        float m = -INFINITY, s = 0.f;
#pragma unroll 1
        for (int c = 0; c < C::COLS; c += 32) {
            uint32_t v[32];
            tmem_ld_32x32b_x32(t_addr + c, v);
            tmem_ld_wait_for(v);
            const int64_t left = p.N - (col0 + c);             // columns of this group inside the vocabulary
            if (left <= 0) continue;
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
        if (row_in && col0 < p.N) p.stats[row * p.stats_ld + col0 / C::COLS] = make_float2(m, s);
    } else {
        int64_t label = -1;
        float lse = 0.f, scale = 0.f;
        bool counts = false;
        if (row_in) {
            const int64_t l = p.labels[row];
            counts = l != p.ignore_index;
            label = l - p.col0 - col0;
            lse = p.lse[row];
            scale = p.scale[row];
        }
#pragma unroll 1
        for (int c = 0; c < C::COLS; c += 64) {
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
            out.put(&tm.c[0], o, col0 + c, row0, warp_in && col0 + c < p.N);
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
template <bool PAIR, bool MN_MAJOR>
__device__ __forceinline__ void mm_load(uint32_t dst, const CUtensorMap* m0, const CUtensorMap* m1, int mn0, int mn1, int k0, uint32_t bar) {
    mm_tma<PAIR>(dst, m0, MN_MAJOR ? mn0 : k0, MN_MAJOR ? k0 : mn0, bar);
    mm_tma<PAIR>(dst + kMmBoxBytes, m1, MN_MAJOR ? mn1 : k0, MN_MAJOR ? k0 : mn1, bar);
}
// First K-step of a range.
__device__ __forceinline__ int mm_split_begin(const MmParams& p, int split) {
    return static_cast<int>(static_cast<int64_t>(p.k_steps) * split / p.splits);
}
// Descriptor of the 16 K-elements from kk * 16 on of a 128-wide operand tile (see umma_smem_desc_sw128).
template <bool MN_MAJOR>
__device__ __forceinline__ uint64_t mm_desc(uint32_t tile, int kk) {
    return MN_MAJOR ? umma_smem_desc_sw128(tile + kk * 2048, kMmBoxBytes, 1024) : umma_smem_desc_sw128(tile + kk * 32, 16, 1024);
}

template <bool PAIR, bool A_MN, bool B_MN, int EPI>
__global__ void __launch_bounds__(kMmThreads, 1)
bf16_mm_kernel(const __grid_constant__ MmMaps tm, const MmParams p) {
    using C = MmCfg<PAIR, EPI>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar_base = smem_base + C::BAR_OFF;
    const uint32_t full = bar_base, empty = full + 8 * C::STAGES;
    const uint32_t acc_full = empty + 8 * C::STAGES, acc_empty = acc_full + 16;
    const uint32_t misc = acc_empty + 16;                  // [0]: TMEM base, [1]: abort flag
    volatile uint32_t* const misc_gen = reinterpret_cast<volatile uint32_t*>(smem_raw + (misc - smem_u32(smem_raw)));

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    Ctx cx{misc_gen + 1, p.error_flag};

    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(acc_full + 8 * i, 1); mbar_init(acc_empty + 8 * i, kMmEpiWarps * (PAIR ? 2 : 1)); }
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

    const int all_n = p.n_tiles * p.n_segs, tiles = p.m_tiles * all_n, total = tiles * p.splits;
    // what a kernel before this one on the stream wrote may be read from here on
    grid_dependency_wait();
    grid_dependency_launch();
    const int unit = PAIR ? blockIdx.x >> 1 : blockIdx.x, units = PAIR ? gridDim.x >> 1 : gridDim.x;

    if (warp == 0) {
        // ================================ TMA producer ================================
        if (elect_one()) {
            Ring r;
            bool ok = true;
            int it = 0;
            for (int tile = unit; ok && tile < total; tile += units, ++it) {
                int mt, nt;
                const int split = tile / tiles, k_begin = mm_split_begin(p, split), k_end = mm_split_begin(p, split + 1);
                tile_coords<8>(tile - split * tiles, p.m_tiles, all_n, mt, nt);
                const int seg = nt >= p.n_tiles ? 1 : 0;
                nt -= seg * p.n_tiles;
                const int m0 = mt * C::TILE_M + static_cast<int>(rank) * 128;
                // where this CTA's two boxes of B start: halves of the gate's and the up projection's columns, or
                // 128 consecutive columns
                const int n0 = C::DUAL ? nt * C::TILE_N : nt * C::TILE_N + static_cast<int>(rank) * 128;
                const int n1 = (C::DUAL && !PAIR) ? n0 : n0 + 64;
                for (int k0 = k_begin; k0 < k_end; ++k0) {
                    int k = serpentine_k(it, k0, k_begin, k_end);
                    const int kseg = k >= p.k_steps0 ? 1 : 0;
                    k -= kseg * p.k_steps0;
                    if (!(ok = wait_bar_t<true, PAIR>(cx, empty + 8 * r.stage, r.phase ^ 1u, 0x001))) break;
                    if (rank == 0) mbar_arrive_expect_tx(full + 8 * r.stage, C::STAGE_BYTES * (PAIR ? 2 : 1));
                    const uint32_t bar = PAIR ? mapa_shared(full + 8 * r.stage, 0) : full + 8 * r.stage;
                    const uint32_t dst = smem_base + r.stage * C::STAGE_BYTES;
                    const int b0 = C::DUAL ? (PAIR ? static_cast<int>(rank) : 0) : (seg | kseg);
                    const int b1 = C::DUAL ? (PAIR ? static_cast<int>(rank) : 1) : (seg | kseg);
                    mm_load<PAIR, A_MN>(dst, &tm.a[kseg], &tm.a[kseg], m0, m0 + 64, k * kMmKStep, bar);
                    mm_load<PAIR, B_MN>(dst + kMmTileBytes, &tm.b[b0], &tm.b[b1], n0, n1, k * kMmKStep, bar);
                    r.advance(C::STAGES);
                }
            }
        }
    } else if (warp == 1) {
        // ================================ UMMA issuer =================================
        if (rank == 0 && elect_one()) {
            constexpr uint32_t idesc = umma_idesc_bf16_f32(PAIR ? 256 : 128, C::BN, A_MN, B_MN);
            Ring r;
            bool ok = true;
            int it = 0;
            for (int tile = unit; ok && tile < total; tile += units, ++it) {
                const int acc = it & 1;
                const uint32_t acc_phase = static_cast<uint32_t>(it >> 1) & 1u;
                // the epilogue has drained this accumulator (the tile before the previous one)
                if (!(ok = wait_bar_t<true, PAIR>(cx, acc_empty + 8 * acc, acc_phase ^ 1u, 0x102))) break;
                const int split = tile / tiles, steps = mm_split_begin(p, split + 1) - mm_split_begin(p, split);
                for (int k = 0; k < steps; ++k) {
                    if (!(ok = wait_bar_t<true, PAIR>(cx, full + 8 * r.stage, r.phase, 0x101))) break;
                    tcgen05_fence_after_sync();
                    const uint32_t as = smem_base + r.stage * C::STAGE_BYTES, bs = as + kMmTileBytes;
#pragma unroll
                    for (int kk = 0; kk < kMmKStep / 16; ++kk) {
                        const uint32_t accumulate = (k > 0 || kk > 0) ? 1u : 0u;
                        if constexpr (PAIR)
                            umma_f16_ss_pair(tmem_base + acc * C::BN, mm_desc<A_MN>(as, kk), mm_desc<B_MN>(bs, kk), idesc, accumulate);
                        else
                            umma_f16_ss(tmem_base + acc * C::BN, mm_desc<A_MN>(as, kk), mm_desc<B_MN>(bs, kk), idesc, accumulate);
                    }
                    if constexpr (PAIR) umma_commit_pair(empty + 8 * r.stage, 3); else umma_commit(empty + 8 * r.stage);
                    r.advance(C::STAGES);
                }
                if (!ok) break;
                if constexpr (PAIR) umma_commit_pair(acc_full + 8 * acc, 3); else umma_commit(acc_full + 8 * acc);
            }
        }
    } else {
        // ================================ epilogue ====================================
        const int q = warp & 3, half = (warp - kMmFirstEpiWarp) >> 2;
        BoxWriter<C::BOXES> out(smem_base + C::BOX_OFF + static_cast<uint32_t>(warp - kMmFirstEpiWarp) * C::BOXES * kEpilogueBoxBytes, lane);
        int it = 0;
        bool ok = true;
        for (int tile = unit; ok && tile < total; tile += units, ++it) {
            int mt, nt;
            const int split = tile / tiles;
            tile_coords<8>(tile - split * tiles, p.m_tiles, all_n, mt, nt);
            const int seg = nt >= p.n_tiles ? 1 : 0;
            nt -= seg * p.n_tiles;
            const int acc = it & 1;
            if (!(ok = wait_bar_t<false, PAIR>(cx, acc_full + 8 * acc, static_cast<uint32_t>(it >> 1) & 1u, 0x201))) break;
            tcgen05_fence_after_sync();
            if (half * C::COLS < C::TILE_N)
                mm_epilogue<C, EPI>(tm, p, out, tmem_base + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(acc * C::BN), half,
                                    static_cast<int64_t>(mt) * C::TILE_M + rank * 128 + q * 32, static_cast<int64_t>(nt) * C::TILE_N, seg, split, lane);
            tcgen05_fence_before_sync();
            __syncwarp();
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

bool operand_map(CUtensorMap* m, const atb::MmOperand& o, bool mn_major, int64_t mn, int64_t K) {
    return make_map_2d(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, o.base, static_cast<uint64_t>(mn_major ? mn : K),
                       static_cast<uint64_t>(mn_major ? K : mn), static_cast<uint64_t>(o.ld) * 2, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B);
}

// Joins the K ranges of a split product: sums of the ranges in their order, then what the epilogue would have done.
// src: [splits][split_rows][cols]; eight columns per thread.
template <int EPI>
__global__ void __launch_bounds__(256) bf16_mm_join_kernel(const MmJoin p) {
    grid_dependency_wait();
    grid_dependency_launch();
    const int64_t per_row = p.N / 8, all = p.M * per_row * p.n_segs;
    const auto sum = [&](int64_t m, int64_t col, float (&v)[8]) {
        const float* src = p.src + m * p.cols + col;
        float4 a = *reinterpret_cast<const float4*>(src), b = *reinterpret_cast<const float4*>(src + 4);
        for (int i = 1; i < p.splits; ++i) {
            src += p.split_rows * p.cols;
            const float4 c = *reinterpret_cast<const float4*>(src), d = *reinterpret_cast<const float4*>(src + 4);
            a.x += c.x; a.y += c.y; a.z += c.z; a.w += c.w;
            b.x += d.x; b.y += d.y; b.z += d.z; b.w += d.w;
        }
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    };
    const auto put = [](void* C, int64_t at, const uint32_t (&o)[4]) {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(C) + at) = make_uint4(o[0], o[1], o[2], o[3]);
    };
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < all; i += static_cast<int64_t>(gridDim.x) * 256) {
        const int64_t m = i / (per_row * p.n_segs), j = i - m * per_row * p.n_segs;
        const int seg = j >= per_row ? 1 : 0;
        const int64_t n = (j - seg * per_row) * 8;
        float v[8];
        sum(m, seg * p.N + n, v);
        uint32_t o[4];
        if constexpr (EPI == atb::kMmStore) {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
            put(p.C[seg], m * p.ldc[seg] + n, o);
        } else if constexpr (EPI == atb::kMmAccumulate) {
            float* dst = p.C32 + m * p.N + n;
#pragma unroll
            for (int e = 0; e < 8; ++e) dst[e] = p.add ? dst[e] + v[e] : v[e];
        } else if constexpr (EPI == atb::kMmGlu) {
            float u[8];
            sum(m, p.N + n, u);
            with_act(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float a0, a1, slope;
                    act_value_slope<act.value>(v[2 * e], a0, slope);
                    act_value_slope<act.value>(v[2 * e + 1], a1, slope);
                    o[e] = pack_bf16(a0 * u[2 * e], a1 * u[2 * e + 1]);
                }
            });
            put(p.C[0], m * p.ldc[0] + n, o);
            if (p.C[1]) {
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                put(p.C[1], m * p.ldc[1] + n, o);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = pack_bf16(u[2 * e], u[2 * e + 1]);
                put(p.C[2], m * p.ldc[2] + n, o);
            }
        } else {
            const uint4 g = *reinterpret_cast<const uint4*>(p.G + m * p.N + n), u = *reinterpret_cast<const uint4*>(p.U + m * p.N + n);
            const uint32_t gw[4] = {g.x, g.y, g.z, g.w}, uw[4] = {u.x, u.y, u.z, u.w};
            uint32_t o2[4];
            with_act(p.act, [&](auto act) {
#pragma unroll
                for (int e = 0; e < 4; ++e) glu_backward_pair<act.value>(gw[e], uw[e], v[2 * e], v[2 * e + 1], o[e], o2[e]);
            });
            put(p.C[0], m * p.ldc[0] + n, o);
            put(p.C[1], m * p.ldc[1] + n, o2);
        }
    }
}

// How a product is laid out on the SMs.
struct MmPlan {
    bool pair;
    int splits;
};

// Cycles of the candidates, by what measured: a K-step of 64 takes 512 cycles in both forms (the pair's 256 x 256 tile is
// bound by the tensor cores; the single CTA's 128 x 128 tile has half the reuse, and its 32 KB per step arrive no
// faster), a work item 2500 more to fill and drain where no other item hides it, and joining the K ranges 4000 for a launch
// and the FP32 sums, written and read once, at 3 KB per cycle.
MmPlan mm_plan(int64_t M, int64_t columns, int64_t k_steps, bool may_split) {
    MmPlan best{false, 1};
    double least = 1e300;
    for (int form = 0; form < 2; ++form) {
        const bool pair = form == 1;
        if (pair && M <= 128) continue;
        const int64_t tile = pair ? 256 : 128, units = pair ? atb::kSmCount / 2 : atb::kSmCount;
        const int64_t tiles = atb::ceil_div(M, tile) * atb::ceil_div(columns, tile);
        for (int s = 1; s <= 16; ++s) {
            if (s > 1 && (!may_split || k_steps / s < 4 || tiles * (s - 1) >= 4 * units)) break;
            const double waves = static_cast<double>(atb::ceil_div(tiles * s, units));
            double t = waves * 512.0 * static_cast<double>(k_steps) / s + 2500.0;
            if (s > 1) t += 4000.0 + 8.0 * s * static_cast<double>(M) * static_cast<double>(columns) / 3000.0;
            if (t < least * 0.98) { least = t; best = {pair, s}; }
        }
    }
    return best;
}
bool can_split(int epilogue) {
    return epilogue == atb::kMmStore || epilogue == atb::kMmAccumulate || epilogue == atb::kMmGlu || epilogue == atb::kMmGluBackward;
}
int64_t accumulator_columns(int epilogue, int64_t N, int n_segs) { return N * (epilogue == atb::kMmGlu ? 2 : n_segs); }
MmPlan plan_of(const atb::MmProblem& q) {
    return mm_plan(q.M, accumulator_columns(q.epilogue, q.N, q.n_segs), atb::ceil_div(q.K, kMmKStep) * q.k_segs, can_split(q.epilogue));
}

template <class... Args>
cudaError_t launch_dependent(void (*kernel)(Args...), unsigned grid, unsigned block, unsigned cluster, size_t smem, cudaStream_t stream, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(block, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;     // may be set up while the kernel before it drains
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// splits > 1: EPI is kMmAccumulate and the sums of the ranges go to q.partial.
template <bool PAIR, bool A_MN, bool B_MN, int EPI>
atb_status_t launch(const atb::MmProblem& q, int splits, const MmDevice& dev, cudaStream_t stream) {
    using C = MmCfg<PAIR, EPI>;
    MmMaps tm;
    MmParams p = {};
    const int n_segs = C::DUAL ? 1 : (q.epilogue == atb::kMmGlu ? 2 : q.n_segs);     // a split gated product: two side by side
    const int n_b = C::DUAL || n_segs == 2 ? 2 : q.k_segs;
    for (int i = 0; i < 2; ++i) {        // a map that is not used is a copy of the first
        if (i >= q.k_segs) tm.a[i] = tm.a[0];
        else if (!operand_map(&tm.a[i], q.A[i], A_MN, q.M, q.K)) return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for A");
        if (i >= n_b) tm.b[i] = tm.b[0];
        else if (!operand_map(&tm.b[i], q.B[i], B_MN, q.N, q.K)) return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for B");
    }
    if constexpr (EPI == atb::kMmAccumulate) {
        float* const base = splits > 1 ? q.partial : q.C32;
        p.split_rows = splits > 1 ? atb::round_up(q.M, 32) : 0;
        p.add = splits > 1 ? 0 : !q.first;
        for (int i = 0; i < n_segs; ++i)      // a map per segment, so that each clips at its own last column
            if (!make_map_2d(&tm.c[i], CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, base + i * q.N, static_cast<uint64_t>(q.N),
                             static_cast<uint64_t>(splits > 1 ? splits * p.split_rows : q.M), static_cast<uint64_t>(q.N * n_segs) * 4, 32, 32,
                             CU_TENSOR_MAP_SWIZZLE_128B))
                return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for the FP32 output");
        if (n_segs == 1) tm.c[1] = tm.c[0];
        tm.c[2] = tm.c[0];
    } else {
        for (int i = 0; i < 3; ++i) {
            if (!q.C[i]) { tm.c[i] = i ? tm.c[0] : tm.a[0]; continue; }              // not written: any valid map
            if (!make_map_2d(&tm.c[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, q.C[i], static_cast<uint64_t>(q.N), static_cast<uint64_t>(q.M),
                             static_cast<uint64_t>(q.ldc[i]) * 2, 64, 32, CU_TENSOR_MAP_SWIZZLE_128B))
                return atb::fail(ATB_ERR_CUDA, "cuTensorMapEncodeTiled failed for an output");
        }
    }
    p.M = q.M; p.N = q.N;
    p.m_tiles = static_cast<int>(atb::ceil_div(q.M, C::TILE_M));
    p.n_tiles = static_cast<int>(atb::ceil_div(q.N, C::TILE_N));
    p.n_segs = n_segs;
    p.k_steps0 = static_cast<int>(atb::ceil_div(q.K, kMmKStep));
    p.k_steps = p.k_steps0 * q.k_segs;
    p.splits = splits;
    p.error_flag = dev.flag;
    p.act = q.act; p.save = q.C[1] != nullptr;
    p.G = static_cast<const __nv_bfloat16*>(q.G); p.U = static_cast<const __nv_bfloat16*>(q.U);
    p.labels = q.labels; p.ignore_index = q.ignore_index; p.col0 = q.col0;
    p.stats = q.stats; p.stats_ld = q.stats_ld; p.label_logit = q.label_logit;
    p.lse = q.lse; p.scale = q.scale;
    const int64_t items = static_cast<int64_t>(p.m_tiles) * p.n_tiles * p.n_segs * splits;
    if (items > (1ll << 30)) return atb::fail(ATB_ERR_BAD_SHAPE, "too many output tiles");
    const int units = PAIR ? dev.sms / 2 : dev.sms;
    const int n_units = static_cast<int>(items < units ? items : units);
    auto kernel = bf16_mm_kernel<PAIR, A_MN, B_MN, EPI>;
    cudaError_t e = cudaSuccess;
    static std::atomic<uint64_t> allowed{0};         // devices on which this kernel has its shared memory allowed
    const uint64_t bit = 1ull << dev.ordinal;
    if (!(allowed.load(std::memory_order_acquire) & bit)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(C::SMEM_BYTES));
        if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
        allowed.fetch_or(bit, std::memory_order_release);
    }
    e = launch_dependent(kernel, static_cast<unsigned>(PAIR ? 2 * n_units : n_units), kMmThreads, PAIR ? 2u : 1u, C::SMEM_BYTES, stream, tm, p);
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "bf16 product launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}

template <bool A_MN, bool B_MN, int EPI>
atb_status_t run(const atb::MmProblem& q, const MmDevice& dev, cudaStream_t stream) {
    const MmPlan plan = plan_of(q);
    if constexpr (EPI == atb::kMmRowStats || EPI == atb::kMmDlogits) {
        return plan.pair ? launch<true, A_MN, B_MN, EPI>(q, 1, dev, stream) : launch<false, A_MN, B_MN, EPI>(q, 1, dev, stream);
    } else {
        if (plan.splits == 1)
            return plan.pair ? launch<true, A_MN, B_MN, EPI>(q, 1, dev, stream) : launch<false, A_MN, B_MN, EPI>(q, 1, dev, stream);
        if (!q.partial) return atb::fail(ATB_ERR_NULL_POINTER, "a product that is split along K needs room for its sums");
        const atb_status_t s = plan.pair ? launch<true, A_MN, B_MN, atb::kMmAccumulate>(q, plan.splits, dev, stream)
                                         : launch<false, A_MN, B_MN, atb::kMmAccumulate>(q, plan.splits, dev, stream);
        if (s != ATB_OK) return s;
        MmJoin j = {};
        j.M = q.M; j.N = q.N; j.n_segs = EPI == atb::kMmGlu ? 1 : q.n_segs;
        j.cols = accumulator_columns(EPI, q.N, q.n_segs);
        j.src = q.partial; j.splits = plan.splits; j.split_rows = atb::round_up(q.M, 32);
        for (int i = 0; i < 3; ++i) { j.C[i] = q.C[i]; j.ldc[i] = q.ldc[i]; }
        j.C32 = q.C32; j.add = !q.first;
        j.act = q.act;
        j.G = static_cast<const __nv_bfloat16*>(q.G); j.U = static_cast<const __nv_bfloat16*>(q.U);
        const int64_t blocks = atb::ceil_div(j.M * (j.N / 8) * j.n_segs, 256), most = static_cast<int64_t>(dev.sms) * 8;
        const cudaError_t e = launch_dependent(bf16_mm_join_kernel<EPI>, static_cast<unsigned>(blocks < most ? blocks : most), 256u, 1u, 0, stream, j);
        if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "bf16 product join launch: %s", cudaGetErrorString(e));
        return ATB_OK;
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
    return ceil_div(N, mm_plan(M, N, ceil_div(K, kMmKStep), false).pair ? 128 : 64);
}

size_t mm_partial_bytes(MmEpilogue epilogue, int64_t M, int64_t N, int64_t K, int k_segs, int n_segs) {
    const int64_t columns = accumulator_columns(epilogue, N, n_segs);
    const MmPlan plan = mm_plan(M, columns, ceil_div(K, kMmKStep) * k_segs, can_split(epilogue));
    return plan.splits > 1 ? static_cast<size_t>(plan.splits) * static_cast<size_t>(round_up(M, 32)) * static_cast<size_t>(columns) * sizeof(float) : 0;
}

atb_status_t mm_launch(const MmProblem& q, cudaStream_t stream) {
    const MmDevice* dev = nullptr;
    const atb_status_t s = mm_device(&dev);
    if (s != ATB_OK) return s;
#define ATB_MM_CASE(LAYOUT, EPI, A_MN, B_MN) \
    if (q.layout == LAYOUT && q.epilogue == EPI) return run<A_MN, B_MN, EPI>(q, *dev, stream);
    ATB_MM_CASE(kMmNN, kMmStore, false, true)
    ATB_MM_CASE(kMmNN, kMmGlu, false, true)
    ATB_MM_CASE(kMmNN, kMmAccumulate, false, true)
    ATB_MM_CASE(kMmNT, kMmStore, false, false)
    ATB_MM_CASE(kMmNT, kMmGluBackward, false, false)
    ATB_MM_CASE(kMmNT, kMmRowStats, false, false)
    ATB_MM_CASE(kMmNT, kMmDlogits, false, false)
    ATB_MM_CASE(kMmTN, kMmStore, true, true)
#undef ATB_MM_CASE
    return fail(ATB_ERR_BAD_ARGUMENT, "no product kernel for layout %d with epilogue %d", static_cast<int>(q.layout), static_cast<int>(q.epilogue));
}

}  // namespace atb
