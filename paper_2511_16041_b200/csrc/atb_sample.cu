// Sampling from logits with temperature, top-k, top-p and min-p from given random numbers (sm_100a).
//
//   weight(l) = 2^((l - max) log2(e) / T), rounded to a multiple of 2^-S;  order: falling logit, rising index
//   kept: the first n words in that order: n <= k;  the weight before a word < p * (weight of the first k);  weight >= min_p
//   token: the first word, in the vocabulary's order, at which the kept weights' sum exceeds u * (all kept weight)
//
// No sort: the kept words are those above a logit tau, and the first c (by index) of those that equal it.  tau is found by
// histograms of counts or weights over ever narrower ranges of logits (512 bins: first of equal width, then of the numbers'
// ordered bit patterns, down to one number), which is 2 to 4 passes over logits that stay in registers.
// Weights are 64-bit integers: their sums are exact, whatever the order they are added in, so that atomics leave no trace and a draw near
// a border falls as it does in 64 bits.
// A cluster of CTAs takes a row, 16 logits a thread: the row is read from memory once, and histograms and sums are joined through
// distributed shared memory.  Rows of more than kMostCtas * 16384 words are read again in every pass.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "atb_internal.h"
#include "dependent_launch.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int kPerThread = 16, kBins = 512, kMostCtas = 8, kMostThreads = 1024, kMostWarps = kMostThreads / 32;
constexpr float kBinsPerUnit = 16.f;       // of the first pass: 32 units below the largest logit, what lies below in the last bin

// A setting: of every row, or one for all.
struct Setting {
    const void* rows;
    double all;
};
struct SampleParams {
    int64_t M, V, ld;
    const void* logits;
    const void* u;
    int u64;
    Setting temperature, top_k, top_p, min_p;      // rows: float, int32, float, float
    int64_t* tokens;
    float* probs;
    int chunks, shift;                             // pieces of 16 logits per thread; S
};

struct Shared {
    uint32_t count[2][kBins];                      // histograms of this CTA, in turn
    unsigned long long weight[2][kBins];
    uint32_t all_count[kBins];                     // of the cluster
    unsigned long long all_weight[kBins];
    float top;                                     // this CTA's largest logit
    unsigned long long total;                      // this CTA's kept weight
    uint32_t equal;                                // this CTA's words at tau
    unsigned long long warp_total[kMostWarps];
    uint32_t warp_equal[kMostWarps];
    float warp_top[kMostWarps];
    // what a pass finds
    int bin;
    unsigned long long above;
    uint32_t above_count, bin_count;
};

__device__ __forceinline__ uint32_t key_of(float l) {            // ordered like the logits; -0 does not occur
    const uint32_t b = __float_as_uint(l);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// -inf for NaN, and +0 for -0, which compare alike.
__device__ __forceinline__ float canonical(float l) { return l == l ? l + 0.f : -INFINITY; }

template <class T>
struct Row {
    static constexpr int VEC = 16 / sizeof(T), NV = kPerThread / VEC;
    const T* row;
    int64_t V, first;                      // first: word of this lane's first element in the warp's first chunk (may lie before the row)
    // word of element e of vector j of chunk c
    __device__ __forceinline__ int64_t word(int c, int j, int e) const { return first + c * (kPerThread * 32) + j * (32 * VEC) + e; }
    __device__ __forceinline__ void load(int c, float (&v)[kPerThread]) const {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int64_t at = word(c, j, 0);
            if (at >= 0 && at + VEC <= V) {
                const uint4 q = __ldg(reinterpret_cast<const uint4*>(row + at));
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    if constexpr (sizeof(T) == 4) v[j * VEC + e] = __uint_as_float(w[e]);
                    else v[j * VEC + e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
                }
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[j * VEC + e] = at + e >= 0 && at + e < V ? static_cast<float>(row[at + e]) : -INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) v[i] = canonical(v[i]);
    }
};

template <class V>
__device__ __forceinline__ V warp_add(V v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
template <class V>
__device__ __forceinline__ V warp_scan(V v, int lane) {          // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V w = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if (lane >= o) v += w;
    }
    return v;
}

// T: type of the logits.  RESIDENT: a thread's logits are 16, and stay in registers.
template <class T, bool RESIDENT>
__global__ void __launch_bounds__(kMostThreads, 1) sample_kernel(const SampleParams p) {
    __shared__ Shared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int64_t m = blockIdx.x / ranks;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, warps = blockDim.x >> 5;
    for (int i = t; i < kBins; i += blockDim.x)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            sh.count[b][i] = 0;
            sh.weight[b][i] = 0;
        }
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();

    Row<T> row;
    row.row = static_cast<const T*>(p.logits) + m * p.ld;
    row.V = p.V;
    {
        // vectors start on 16-byte boundaries: positions are counted from the one at or below the row's first word
        const int64_t skip = static_cast<int64_t>(reinterpret_cast<uintptr_t>(row.row) & 15u) / static_cast<int64_t>(sizeof(T));
        row.first = (static_cast<int64_t>(rank) * warps + warp) * p.chunks * (kPerThread * 32) + lane * Row<T>::VEC - skip;
    }
    float kept_in_registers[kPerThread];
    if constexpr (RESIDENT) row.load(0, kept_in_registers);
    // f(chunk, logits) over this thread's logits
    const auto each = [&](auto&& f) {
        if constexpr (RESIDENT) {
            f(0, kept_in_registers);
        } else {
#pragma unroll 1
            for (int c = 0; c < p.chunks; ++c) {
                float v[kPerThread];
                row.load(c, v);
                f(c, v);
            }
        }
    };

    // ---- the row's settings
    const auto real = [&](const Setting& s) { return s.rows ? static_cast<double>(static_cast<const float*>(s.rows)[m]) : s.all; };
    const double temperature = real(p.temperature), top_p = real(p.top_p), min_p = real(p.min_p);
    int64_t k = p.top_k.rows ? static_cast<const int32_t*>(p.top_k.rows)[m] : static_cast<int64_t>(p.top_k.all);
    double u = p.u64 ? static_cast<const double*>(p.u)[m] : static_cast<double>(static_cast<const float*>(p.u)[m]);
    const bool greedy = !(temperature > 0.0);
    if (greedy) k = 1;
    if (k <= 0 || k > p.V) k = p.V;
    const double slope = greedy ? 1.4426950408889634074 : 1.4426950408889634074 / temperature;
    // weight >= min_p by the exponents; 1 and more keep what weighs 1 in 64 bits, which is more than 1 - 2^-54
    const double deepest = min_p > 0.0 ? fmax(min_p < 1.0 ? -log2(min_p) : 0.0, 0x1p-54 * 1.4426950408889634074) : INFINITY;

    // ---- the largest logit
    float top = -INFINITY;
    each([&](int, const float (&v)[kPerThread]) {
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) top = fmaxf(top, v[i]);
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if (lane == 0) sh.warp_top[warp] = top;
    __syncthreads();
    if (warp == 0) {
        top = lane < warps ? sh.warp_top[lane] : -INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (lane == 0) sh.top = top;
    }
    cluster.sync();
    for (int r = 0; r < ranks; ++r) top = fmaxf(r ? top : -INFINITY, *cluster.map_shared_rank(&sh.top, r));
    if (top == -INFINITY) {                // nothing to draw from: the same for the whole cluster
        if (rank == 0 && t == 0) {
            p.tokens[m] = -1;
            if (p.probs) p.probs[m] = 0.f;
        }
        cluster.sync();
        return;
    }

    // depth of a logit below the largest, in powers of 2
    const auto depth = [&](float l) { return l == top ? 0.0 : (static_cast<double>(top) - static_cast<double>(l)) * slope; };
    const auto weight = [&](float l) -> unsigned long long {
        const double y = depth(l);
        return y < p.shift + 2 ? __double2ull_rn(exp2(static_cast<double>(p.shift) - y)) : 0ull;
    };
    const auto bin_of = [&](float l) {     // falls with l, as every step of it does
        const float d = (top - l) * kBinsPerUnit;
        return l == top ? 0 : d < static_cast<float>(kBins - 1) ? static_cast<int>(d) : kBins - 1;
    };

    // ---- the kept words: above tau, and `quota` of those that equal it
    uint32_t tau = 0;                      // key; nothing that can be drawn is at 0
    uint32_t quota = 0, equal_all = 0;     // equal_all: words at tau
    int turn = 0;
    // One search: the first number, from the largest logit down, at which the sum (of counts, or of weights, over the words that `in` admits)
    // reaches `goal`.
    const auto search = [&](bool by_weight, auto&& reached, auto&& admits) {
        // the words looked at: the first pass's bin, and keys low .. high
        int bin = -1;
        uint32_t low = 0, high = 0xFFFFFFFFu;
        int width = 0;                     // a bin holds 2^width keys
        unsigned long long above = 0;
        uint32_t above_count = 0;
        while (true) {
            each([&](int, const float (&v)[kPerThread]) {
#pragma unroll
                for (int i = 0; i < kPerThread; ++i) {
                    const uint32_t key = key_of(v[i]);
                    if (v[i] == -INFINITY || !admits(key)) continue;
                    int b = bin_of(v[i]);
                    if (bin >= 0) {
                        if (b != bin || key < low || key > high) continue;
                        b = static_cast<int>((high - key) >> width);
                    }
                    atomicAdd(&sh.count[turn][b], 1u);
                    if (by_weight) atomicAdd(&sh.weight[turn][b], weight(v[i]));
                }
            });
            cluster.sync();
            for (int i = t; i < kBins; i += blockDim.x) {
                uint32_t n = 0;
                unsigned long long w = 0;
                for (int r = 0; r < ranks; ++r) {
                    const Shared* other = cluster.map_shared_rank(&sh, r);
                    n += other->count[turn][i];
                    if (by_weight) w += other->weight[turn][i];
                }
                sh.all_count[i] = n;
                sh.all_weight[i] = w;
                // the histogram of the pass before, which nobody reads any more, is the next one's
                sh.count[turn ^ 1][i] = 0;
                sh.weight[turn ^ 1][i] = 0;
            }
            __syncthreads();
            if (warp == 0) {
                // a lane has 16 bins; it reads them from another one on than its neighbours (banks)
                constexpr int PER = kBins / 32;
                uint32_t n = 0;
                unsigned long long w = 0;
                for (int i = 0; i < PER; ++i) {
                    const int b = lane * PER + ((i + lane) & (PER - 1));
                    n += sh.all_count[b];
                    w += sh.all_weight[b];
                }
                const uint32_t n_to = warp_scan(n, lane);
                const unsigned long long w_to = warp_scan(w, lane);
                const unsigned here = __ballot_sync(0xFFFFFFFFu, reached(above_count + n_to, above + w_to));
                if (here == 0) {
                    if (lane == 0) sh.bin = -1;
                } else if (lane == __ffs(here) - 1) {
                    uint32_t cn = above_count + n_to - n;
                    unsigned long long cw = above + w_to - w;
                    int b = lane * PER;
                    for (; b < lane * PER + PER - 1; ++b) {
                        if (reached(cn + sh.all_count[b], cw + sh.all_weight[b])) break;
                        cn += sh.all_count[b];
                        cw += sh.all_weight[b];
                    }
                    sh.bin = b;
                    sh.above_count = cn;
                    sh.above = cw;
                    sh.bin_count = sh.all_count[b];
                }
            }
            __syncthreads();
            turn ^= 1;
            const int found = sh.bin;
            above = sh.above;
            above_count = sh.above_count;
            const uint32_t in_bin = sh.bin_count;
            __syncthreads();               // sh.bin is written again
            if (found < 0) return false;   // not reached by all of them
            if (bin < 0) {
                // keys of the bin's words: its ends, and more than the roundings of bin_of and of the ends can be
                bin = found;
                const float up = static_cast<float>(found) / kBinsPerUnit, down = static_cast<float>(found + 1) / kBinsPerUnit;
                const float slack = (fabsf(top) + down) * 0x1p-22f;
                high = found == 0 ? key_of(top) : key_of(canonical(fminf(top, top - up + slack)));
                low = found == kBins - 1 ? 0u : key_of(canonical(top - down - slack));
                if (!(top < INFINITY)) {   // an infinite logit stands alone, all others are in the last bin
                    high = found == 0 ? key_of(top) : key_of(top) - 1u;
                    low = found == 0 ? high : 0u;
                }
            } else if (width == 0) {
                tau = high - static_cast<uint32_t>(found);
                equal_all = in_bin;
                quota = in_bin;
                return true;
            } else {
                high -= static_cast<uint32_t>(found) << width;
                const uint32_t span = (1u << width) - 1u;
                if (high - low > span) low = high - span;
            }
            const uint32_t keys = high - low;
            width = 0;
            while ((keys >> width) >= kBins) ++width;
        }
    };

    if (k < p.V) {
        if (search(false, [&](uint32_t n, unsigned long long) { return n >= static_cast<uint64_t>(k); }, [](uint32_t) { return true; }))
            quota = static_cast<uint32_t>(k - sh.above_count);
    }
    __syncthreads();
    if (top_p < 1.0 && !greedy) {
        const uint32_t tau_k = tau, quota_k = quota, equal_k = equal_all;
        // the weight of the first k: all above tau, and `quota` times tau's own
        unsigned long long mine = 0;
        each([&](int, const float (&v)[kPerThread]) {
#pragma unroll
            for (int i = 0; i < kPerThread; ++i)
                if (key_of(v[i]) > tau_k) mine += weight(v[i]);
        });
        mine = warp_add(mine);
        if (lane == 0) sh.warp_total[warp] = mine;
        __syncthreads();
        if (warp == 0) {
            mine = warp_add(lane < warps ? sh.warp_total[lane] : 0ull);
            if (lane == 0) sh.total = mine;
        }
        cluster.sync();
        unsigned long long sum = 0;
        for (int r = 0; r < ranks; ++r) sum += *cluster.map_shared_rank(&sh.total, r);
        const unsigned long long at_tau = tau_k ? weight(of_key(tau_k)) : 0ull;
        const double whole = static_cast<double>(sum + quota_k * at_tau), goal = top_p > 0.0 ? top_p * whole : 0.0;
        // the words that equal tau count all here: where they take the sum to the goal, `quota` is cut below
        const bool found = search(true, [&](uint32_t n, unsigned long long w) { return n > 0 && static_cast<double>(w) >= goal; }, [&](uint32_t key) { return key >= tau_k; });
        if (found) {
            // of the words at tau, those before which the weight is below the goal
            const double before = static_cast<double>(sh.above), each_one = static_cast<double>(weight(of_key(tau)));
            const double n = goal > before ? ceil((goal - before) / each_one) : 0.0;
            quota = n < 1.0 ? 1u : n < static_cast<double>(equal_all) ? static_cast<uint32_t>(n) : equal_all;
            if (tau == tau_k && quota > quota_k) quota = quota_k;
        } else {
            tau = tau_k;
            quota = quota_k;
            equal_all = equal_k;
        }
        __syncthreads();
    }

    // ---- the draw
    // words at tau before this warp's, where not all are kept
    const bool ranked = quota < equal_all;
    uint32_t equals_before = 0;
    if (ranked) {
        uint32_t n = 0;
        each([&](int, const float (&v)[kPerThread]) {
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) n += key_of(v[i]) == tau;
        });
        n = warp_add(n);
        if (lane == 0) sh.warp_equal[warp] = n;
        __syncthreads();
        if (warp == 0) {
            n = lane < warps ? sh.warp_equal[lane] : 0u;
            const uint32_t to = warp_scan(n, lane);
            if (lane < warps) sh.warp_equal[lane] = to - n;
            if (lane == 31) sh.equal = to;
        }
        cluster.sync();
        for (int r = 0; r < rank; ++r) equals_before += *cluster.map_shared_rank(&sh.equal, r);
        equals_before += sh.warp_equal[warp];
    }
    // f(chunk, vector, weights of its elements) over the warp's vectors in the words' order, weight 0 for what is not kept
    constexpr int VEC = Row<T>::VEC, NV = Row<T>::NV;
    const auto walk = [&](auto&& f) {
        uint32_t before = equals_before;
        each([&](int c, const float (&v)[kPerThread]) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                uint32_t rank_here = 0;
                if (ranked) {
                    uint32_t n = 0;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) n += key_of(v[j * VEC + e]) == tau;
                    const uint32_t to = warp_scan(n, lane);
                    rank_here = before + to - n;
                    before += __shfl_sync(0xFFFFFFFFu, to, 31);
                }
                unsigned long long w[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float l = v[j * VEC + e];
                    const uint32_t key = key_of(l);
                    bool in = key > tau;
                    if (key == tau) in = !ranked || rank_here++ < quota;
                    w[e] = in && l > -INFINITY && depth(l) <= deepest ? weight(l) : 0ull;
                }
                f(c, j, w);
            }
        });
    };
    unsigned long long mine = 0;
    walk([&](int, int, const unsigned long long (&w)[VEC]) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) mine += w[e];
    });
    mine = warp_add(mine);
    if (lane == 0) sh.warp_total[warp] = mine;
    __syncthreads();
    if (warp == 0) {
        const unsigned long long own = lane < warps ? sh.warp_total[lane] : 0ull, to = warp_scan(own, lane);
        if (lane < warps) sh.warp_total[lane] = to - own;
        if (lane == 31) sh.total = to;
    }
    cluster.sync();
    unsigned long long base = 0, all = 0;
    for (int r = 0; r < ranks; ++r) {
        const unsigned long long v = *cluster.map_shared_rank(&sh.total, r);
        if (r < rank) base += v;
        all += v;
    }
    base += sh.warp_total[warp];
    // the first word whose sum exceeds u * all: at least `target`
    if (!(u > 0.0)) u = 0.0;
    const double at = u * static_cast<double>(all);
    const unsigned long long target = (at < static_cast<double>(all) ? min(static_cast<unsigned long long>(at), all - 1) : all - 1) + 1;
    if (base < target && target <= base + mine) {                // this warp has it
        unsigned long long before = base;
        bool done = false;
        walk([&](int c, int j, const unsigned long long (&w)[VEC]) {
            unsigned long long own = 0;
#pragma unroll
            for (int e = 0; e < VEC; ++e) own += w[e];
            const unsigned long long to = warp_scan(own, lane) + before;
            before = __shfl_sync(0xFFFFFFFFu, to, 31);
            if (!done && to >= target && to - own < target) {
                unsigned long long run = to - own;
                int word = 0;
                unsigned long long its = 0;
                bool found = false;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    run += w[e];
                    if (!found && run >= target) { found = true; word = e; its = w[e]; }
                }
                p.tokens[m] = row.word(c, j, word);
                if (p.probs) p.probs[m] = static_cast<float>(static_cast<double>(its) / static_cast<double>(all));
                done = true;
            }
        });
    }
    cluster.sync();                        // nobody leaves while its sums may still be read
}

bool known_type(int t) { return t == ATB_F32 || t == ATB_BF16; }
bool aligned_to(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }

template <class T>
cudaError_t launch(SampleParams p, cudaStream_t st) {
    const int64_t positions = p.V + 16 / static_cast<int64_t>(sizeof(T)) - 1;       // a row may start inside a vector
    const int64_t threads = atb::ceil_div(positions, kPerThread);
    int ctas = 1;
    while (ctas < kMostCtas && threads > static_cast<int64_t>(ctas) * kMostThreads) ctas *= 2;
    p.chunks = static_cast<int>(atb::ceil_div(threads, static_cast<int64_t>(ctas) * kMostThreads));
    int block = static_cast<int>(atb::round_up(atb::ceil_div(threads, static_cast<int64_t>(ctas) * p.chunks), 32));
    if (block < 64) block = 64;
    int log2v = 0;
    while ((1ll << log2v) < p.V) ++log2v;
    p.shift = 62 - log2v < 45 ? 62 - log2v : 45;
    const unsigned grid = static_cast<unsigned>(p.M * ctas);
    return p.chunks == 1 ? atb::launch_dependent(sample_kernel<T, true>, grid, static_cast<unsigned>(block), static_cast<unsigned>(ctas), 0, st, p)
                         : atb::launch_dependent(sample_kernel<T, false>, grid, static_cast<unsigned>(block), static_cast<unsigned>(ctas), 0, st, p);
}

}  // namespace

extern "C" atb_status_t atb_sample(int64_t M, int64_t V, int type, const void* logits_dev, int64_t ld, int u_type, const void* u_dev, double temperature,
                                   const float* temperature_dev, int64_t top_k, const int32_t* top_k_dev, double top_p, const float* top_p_dev, double min_p,
                                   const float* min_p_dev, int64_t* tokens_dev, float* probs_dev, void* stream) {
    atb::clear_error();
    if (!known_type(type)) return atb::fail(ATB_ERR_BAD_ARGUMENT, "type=%d: ATB_F32 or ATB_BF16", type);
    if (u_type != ATB_F32 && u_type != ATB_F64) return atb::fail(ATB_ERR_BAD_ARGUMENT, "u_type=%d: ATB_F32 or ATB_F64", u_type);
    if (!temperature_dev && !(temperature >= 0.0)) return atb::fail(ATB_ERR_BAD_ARGUMENT, "temperature must be >= 0");
    if ((!top_p_dev && !(top_p == top_p)) || (!min_p_dev && !(min_p == min_p))) return atb::fail(ATB_ERR_BAD_ARGUMENT, "top_p and min_p must be numbers");
    if (M < 0 || V < 1 || M > (1ll << 27) || V > (1ll << 30)) return atb::fail(ATB_ERR_BAD_SHAPE, "need 0 <= M <= 2^27 and 1 <= V <= 2^30 (got %lld, %lld)", (long long)M, (long long)V);
    if (M == 0) return ATB_OK;
    if (!logits_dev || !u_dev || !tokens_dev) return atb::fail(ATB_ERR_NULL_POINTER, "the logits, u and the tokens must be non-NULL");
    if (M > 1 && ld < V) return atb::fail(ATB_ERR_BAD_SHAPE, "ld=%lld must be >= V", (long long)ld);
    if (!aligned_to(logits_dev, type == ATB_F32 ? 4 : 2) || !aligned_to(u_dev, u_type == ATB_F64 ? 8 : 4) || !aligned_to(temperature_dev, 4) || !aligned_to(top_k_dev, 4) ||
        !aligned_to(top_p_dev, 4) || !aligned_to(min_p_dev, 4) || !aligned_to(tokens_dev, 8) || !aligned_to(probs_dev, 4))
        return atb::fail(ATB_ERR_MISALIGNED, "every pointer must be aligned to its elements");
    int sms = 0;
    const atb_status_t s = atb::op_device(&sms);
    if (s != ATB_OK) return s;
    SampleParams p = {};
    p.M = M; p.V = V; p.ld = ld;
    p.logits = logits_dev;
    p.u = u_dev; p.u64 = u_type == ATB_F64;
    p.temperature = {temperature_dev, temperature};
    p.top_k = {top_k_dev, static_cast<double>(top_k < 0 ? 0 : top_k > V ? V : top_k)};
    p.top_p = {top_p_dev, top_p};
    p.min_p = {min_p_dev, min_p};
    p.tokens = tokens_dev; p.probs = probs_dev;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = type == ATB_F32 ? launch<float>(p, st) : launch<__nv_bfloat16>(p, st);
    if (e != cudaSuccess) return atb::fail(ATB_ERR_CUDA, "sampling launch: %s", cudaGetErrorString(e));
    return ATB_OK;
}
