// Sampling from logits with temperature, top-k, top-p and min-p from given random numbers (sm_100a).
//
//   weight(l) = 2^((l - max) log2(e) / T), rounded to a multiple of 2^-S;  order: falling logit, rising index
//   kept: the first n words in that order: n <= k;  the weight before a word < p * (weight of the first k);  weight >= min_p
//   token: the first word, in the vocabulary's order, at which the kept weights' sum exceeds u * (all kept weight)
//
// Weights are 64-bit integers: their sums are exact, whatever the order they are added in, so that atomics leave no trace.  What is rounded
// is each weight, by 2^-(S + 1) of the largest at most (S = 45 up to 131072 words): a border falls otherwise than with sums in 64 bits where
// it is within that, summed over the words, of a word's weight: 5 of 7.4 million rows of 131072 words at p = 0.99, by one word each, which
// are the rows that these rounded weights give.  The row is not sorted: the kept words are those above a logit tau, and the first c (by index) of
// those that equal it.
//   few words at most (k up to 3/4 of 256): the k-th largest of 256 groups' largest logits is at most the k-th largest logit, so that the
//     words that reach it are few (about 60 for k = 50): one CTA ranks those and draws
//   else tau is found by histograms over ever narrower ranges of logits (1024 bins: first of equal width, then of the numbers' ordered bit
//     patterns, down to one number), of counts for top-k; for top-p a first histogram of counts bounds the weight in its bins, so that only
//     the few bins that the border may be in are looked at word by word
// A cluster of CTAs takes a row, 32 logits a thread in shared memory: the row is read from memory once, and histograms and sums are
// joined through distributed shared memory.  Rows of more than kMostCtas * 16384 words are read again in every pass.
// Bound by instructions and by the waits of a cluster's CTAs for one another.  A row's load, maximum, waits and exit follow one another, with the other
// row on the SM to cover them: 512 rows of 131072 words are 14 rounds of 37 clusters, and the greedy draw, which needs the maximum and
// its place, takes 218 us.  top-p takes about 100 instructions a word (one exact weight
// is 21, the bounds' approximate weight and count 20) and seven waits; two CTAs of different rows share an SM, so that one works
// while the other waits.  131072 words, FP32: one row, k = 50, 12 us, plain temperature 13 us, top-p 30 us; 512 rows 262, 282 and 560 us (the
// logits are 41 us of memory traffic).  Logits in registers, 16 of 1024 threads and loops unrolled over them, took 250 instructions
// a word (what a warp does once per pass counted for half as many words) and 1410 us; branches around the sums of weights, 30 us.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "atb_internal.h"
#include "dependent_launch.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int kVectors = 8, kPerThread = 4 * kVectors, kBins = 1024, kMostCtas = 8, kMostThreads = 512, kMostWarps = kMostThreads / 32;
constexpr float kBinsPerUnit = 32.f;       // of the first pass: 32 units below the largest logit, what lies below in the last bin

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
    int chunks, shift;                             // pieces of 4 * vectors logits per thread; S
    int vectors;                                   // even
    int group;                                     // lanes that share a largest logit
};
static_assert(kBins == 1024, "32 spans of 32 bins: a lane to a span");
constexpr int kMostGroups = 256, kCandidates = 512, kWords = 2048, kSpans = kBins / 32;
struct Candidate {
    float l;
    int word;
};
// What the row's first CTA has found, for all.
struct Found {
    int first, last;                               // bins; first -1: the goal is not reached
    uint32_t active, above_count;                  // words in those bins, words above them
    uint32_t tau, equal;                           // where done: the number, and the words that equal it
    int done;
    unsigned long long above;                      // weight above them
    double goal;
};
struct FewWords {                                  // all candidates; the first k of them in their order
    Candidate all[kCandidates], kept[kCandidates];
    unsigned long long weight[kCandidates];
};
struct Shared {
    union {                                        // the first CTA's, when it goes on alone
        FewWords few;
        float words[kWords];
    };
    union {                                        // this CTA's
        Candidate candidate[kCandidates];
        Candidate active[kWords];
    };
    uint32_t candidates, listed;                   // of either; of the last list
    uint32_t count[kBins];                         // histogram
    unsigned long long weight[kBins];
    uint32_t span_count[kSpans];                   // sums over 32 bins
    unsigned long long span_weight[kSpans];
    float span_most[kSpans], span_least[kSpans], most, least;
    Found found;
    unsigned long long beyond, whole;              // weight above the bins looked at, of all words
    double real;                                   // this CTA's weight, about
    double warp_real[kMostWarps];
    float group_top[kMostGroups];                  // this CTA's groups' largest logits
    float all_groups[kMostGroups];
    float floor;
    float top;                                     // this CTA's largest logit, and the row's
    float row_top;
    unsigned long long total;                      // this CTA's kept weight
    unsigned long long base, all;                  // that of the CTAs before this one, of all
    uint32_t equal;                                // this CTA's words at tau
    uint32_t joined;                               // a sum over the cluster
    uint32_t ends[kMostCtas];                      // of the CTAs' words in the first one's list
    float lanes[32];                               // the last words of a search
    unsigned long long warp_total[kMostWarps];
    unsigned long long warp_beyond[kMostWarps];
    uint32_t warp_equal[kMostWarps];
    float warp_top[kMostWarps];
    double u, top_p, deepest;                      // the row's; deepest: powers of 2 below the largest that min_p leaves
    double table[16];                              // 2^(S - j / 16)
};

__device__ __forceinline__ uint32_t key_of(float l) {            // ordered like the logits; -0 does not occur
    const uint32_t b = __float_as_uint(l);
    return b ^ (static_cast<uint32_t>(static_cast<int32_t>(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// -inf for NaN, and +0 for -0, which compare alike.
__device__ __forceinline__ float canonical(float l) {
    float v;
    asm("max.f32 %0, %1, 0fFF800000;" : "=f"(v) : "f"(l + 0.f));
    return v;
}

// A warp's logits: chunks of 128 * vectors consecutive words, in shared memory as vectors of 4, vector j of lane i at words 128 j + 4 i of the chunk.
template <class T>
struct Row {
    const T* row;
    int V, vectors, first;                 // first: word of the warp's first logit (may lie before the row)
    bool alone;                            // logits that are not `only` become -inf, those that are 0
    float only;
    // word of element e of this lane's vector j of chunk c
    __device__ __forceinline__ int word(int c, int j, int lane, int e) const { return first + (c * vectors + j) * 128 + lane * 4 + e; }
    __device__ __forceinline__ float taken(float l) const {
        const float v = canonical(l);
        return !alone ? v : v == only ? 0.f : -INFINITY;
    }
    // Chunk c to `to`, this warp's place; returns this lane's largest.  Vectors of 16 bytes that lie inside the row are loaded whole.
    __device__ __forceinline__ float load(int c, float4* to, int lane) const {
        float top = -INFINITY;
        constexpr int PER = 16 / sizeof(T), AT_ONCE = 16 / PER, STEP = AT_ONCE * PER / 4;      // loads in flight, of STEP vectors
        const int from = first + c * vectors * 128 + lane * PER;
        __syncwarp();                      // the warp has read the chunk before
#pragma unroll 1
        for (int j = 0; j < vectors; j += STEP) {
            uint4 q[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                const int at = j + i * PER / 4 < vectors ? from + j * 128 + i * 32 * PER : V;
                if (at >= 0 && at <= V - PER) {
                    q[i] = __ldg(reinterpret_cast<const uint4*>(row + at));
                } else {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (sizeof(T) == 4) {
                            w[e] = at + e >= 0 && at + e < V ? reinterpret_cast<const uint32_t*>(row)[at + e] : 0xFF800000u;
                        } else {
                            const auto one = [&](int a) -> uint32_t { return a >= 0 && a < V ? reinterpret_cast<const uint16_t*>(row)[a] : 0xFF80u; };
                            w[e] = one(at + 2 * e) | one(at + 2 * e + 1) << 16;
                        }
                    }
                    q[i] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                if (j + i * PER / 4 >= vectors) continue;
                const uint32_t w[4] = {q[i].x, q[i].y, q[i].z, q[i].w};
                float4* const dst = to + (j * 128 + i * 32 * PER + lane * PER) / 4;
                if constexpr (sizeof(T) == 4) {
                    const float4 v = make_float4(taken(__uint_as_float(w[0])), taken(__uint_as_float(w[1])), taken(__uint_as_float(w[2])), taken(__uint_as_float(w[3])));
                    *dst = v;
                    top = fmaxf(top, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const auto at = [&](int e) { return taken(__uint_as_float(e & 1 ? w[2 * h + e / 2] & 0xFFFF0000u : w[2 * h + e / 2] << 16)); };
                        const float4 v = make_float4(at(0), at(1), at(2), at(3));
                        dst[h] = v;
                        top = fmaxf(top, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
                    }
                }
            }
        }
        __syncwarp();
        return top;
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

// 2^(S - d slope), d >= 0, to the nearest integer, where slope16 = 16 slope: 2^(-round(16 y) / 16), from a table times 2^S, and the rest, at
// most 2^-5, by the first terms of its series (Tang's table-driven method), relative error below 2^-50.  The sums with
// 1.5 * 2^52 and 2^52 round to an integer.  Sixteen entries lie in banks of their own; the series' terms are operands from constant
// memory.  d slope < 1060.  As a double, and with 2^52 added, whose bits are the integer's.
constexpr double kLn2of16 = 0.69314718055994530942 / 16;
__constant__ double kSeries[6] = {kLn2of16,
                                  kLn2of16* kLn2of16 / 2,
                                  kLn2of16* kLn2of16* kLn2of16 / 6,
                                  kLn2of16* kLn2of16* kLn2of16* kLn2of16 / 24,
                                  kLn2of16* kLn2of16* kLn2of16* kLn2of16* kLn2of16 / 120,
                                  kLn2of16* kLn2of16* kLn2of16* kLn2of16* kLn2of16* kLn2of16 / 720};
__constant__ double kRound[2] = {0x1.8p52, 0x1p52};
__device__ __forceinline__ double fixed_exp2_biased(double d, double slope16, const double* table) {
    const double near = fma(d, slope16, kRound[0]);
    const int n = __double2loint(near);
    const double r = fma(-d, slope16, near - kRound[0]);         // 16 y = n - r
    double p = fma(r, kSeries[5], kSeries[4]);
#pragma unroll
    for (int i = 3; i >= 0; --i) p = fma(r, p, kSeries[i]);
    p = fma(r, p, 1.0) * table[n & 15];
    return __hiloint2double(__double2hiint(p) - (n & ~15) * 65536, __double2loint(p)) + kRound[1];
}

// Sum over the first `ranks` CTAs of what they have at `own`: by one warp, a lane to a CTA, so that a value crosses once.
template <class V>
__device__ __forceinline__ V cluster_sum(const cg::cluster_group& cluster, int ranks, V* own, int lane) {
    return warp_add(lane < ranks ? *cluster.map_shared_rank(own, lane) : V(0));
}

// T: type of the logits.  RESIDENT: a row's logits fit the cluster's shared memory.
template <class T, bool RESIDENT>
__global__ void __launch_bounds__(kMostThreads, 2) sample_kernel(const SampleParams p) {
    __shared__ Shared sh;
    extern __shared__ float4 logits[];     // [warps][32 vectors]
    cg::cluster_group cluster = cg::this_cluster();
    const int ranks = static_cast<int>(cluster.num_blocks()), rank = static_cast<int>(cluster.block_rank());
    const int64_t m = blockIdx.x / ranks;
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5, warps = blockDim.x >> 5;
    for (int i = t; i < kBins; i += blockDim.x) {
        sh.count[i] = 0;
        sh.weight[i] = 0;
    }
    if (t == 0) sh.candidates = 0;
    if (t < 16) sh.table[t] = exp2(p.shift - t * 0.0625);
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();

    Row<T> row;
    row.row = static_cast<const T*>(p.logits) + m * p.ld;
    row.V = static_cast<int>(p.V);
    {
        // vectors start on 16-byte boundaries: positions are counted from the one at or below the row's first word
        const int64_t skip = static_cast<int64_t>(reinterpret_cast<uintptr_t>(row.row) & 15u) / static_cast<int64_t>(sizeof(T));
        row.vectors = p.vectors;
        row.first = (rank * warps + warp) * p.chunks * p.vectors * 128 - static_cast<int>(skip);
    }
    row.alone = false;
    row.only = 0.f;
    float4* const mine4 = logits + warp * 32 * p.vectors;
    float top = -INFINITY;
    if constexpr (RESIDENT) {
        top = row.load(0, mine4, lane);
    } else {
#pragma unroll 1
        for (int c = 0; c < p.chunks; ++c) top = fmaxf(top, row.load(c, mine4, lane));
    }
    // f(chunk, vector, logits) over this thread's logits in the words' order
    const auto each = [&](auto&& f) {
#pragma unroll 1
        for (int c = 0; c < (RESIDENT ? 1 : p.chunks); ++c) {
            if constexpr (!RESIDENT) row.load(c, mine4, lane);
#pragma unroll 1
            for (int j = 0; j < p.vectors; ++j) {
                const float4 q = mine4[j * 32 + lane];
                const float v[4] = {q.x, q.y, q.z, q.w};
                f(c, j, v);
            }
        }
    };

    // ---- the row's settings
    const auto real = [&](const Setting& s) { return s.rows ? static_cast<double>(static_cast<const float*>(s.rows)[m]) : s.all; };
    const double temperature = real(p.temperature);
    int64_t k = p.top_k.rows ? static_cast<const int32_t*>(p.top_k.rows)[m] : static_cast<int64_t>(p.top_k.all);
    const bool greedy = !(temperature > 0.0);
    if (greedy) k = 1;
    if (k <= 0 || k > p.V) k = p.V;
    double slope = greedy ? 1.4426950408889634074 : 1.4426950408889634074 / temperature;
    if (t == 0) {                          // what is needed late waits in shared memory
        const double min_p = real(p.min_p), top_p = real(p.top_p);
        sh.u = p.u64 ? static_cast<const double*>(p.u)[m] : static_cast<double>(static_cast<const float*>(p.u)[m]);
        sh.top_p = greedy ? 1.0 : top_p < 0.0 ? 0.0 : top_p;     // (-inf times no weight would be NaN)
        // weight >= min_p by the exponents; 1 and more keep what weighs 1 in 64 bits, which is more than 1 - 2^-54
        sh.deepest = min_p > 0.0 ? fmax(min_p < 1.0 ? -log2(min_p) : 0.0, 0x1p-54 * 1.4426950408889634074) : INFINITY;
    }

    // ---- the largest logit, and those of the groups
    for (int o = 1; o < 32; o <<= 1) {
        if (o == p.group && !(lane & (o - 1))) sh.group_top[t / o] = top;
        top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    }
    if (p.group == 32 && lane == 0) sh.group_top[warp] = top;
    if (lane == 0) sh.warp_top[warp] = top;
    __syncthreads();
    if (warp == 0) {
        top = lane < warps ? sh.warp_top[lane] : -INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (lane == 0) sh.top = top;
    }
    cluster.sync();
    if (warp == 0) {
        top = lane < ranks ? *cluster.map_shared_rank(&sh.top, lane) : -INFINITY;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (lane == 0) sh.row_top = top;
    }
    __syncthreads();
    top = sh.row_top;
    if (top == -INFINITY) {                // nothing to draw from: the same for the whole cluster
        if (rank == 0 && t == 0) {
            p.tokens[m] = -1;
            if (p.probs) p.probs[m] = 0.f;
        }
        cluster.sync();
        return;
    }

    // Where only words that equal the largest weigh anything - it is infinite, or its neighbour is more than 250 powers of 2 below it - the others
    // become -inf and those 0, so that all differences below are finite and no product of them is too large.
    const double nearest = fmax(static_cast<double>(fabsf(top)) * 0x1p-24, 0x1p-149);         // no two numbers at the largest are nearer
    const bool alone = !(top < INFINITY) || !(slope * nearest <= 250.0);
    if (alone) {
        row.alone = true;
        row.only = top;
        top = 0.f;
        slope = 1.0;
        if constexpr (RESIDENT) row.load(0, mine4, lane);
    }
    // depth of a logit below the largest, in powers of 2
    const auto depth = [&](float l) { return (static_cast<double>(top) - static_cast<double>(l)) * slope; };
    const float half_top = 0.5f * top, slope_f = fminf(static_cast<float>(slope), 1e30f);
    const double slope16 = 16.0 * slope, top64 = top;
    // no logit deeper than this weighs anything, and neither does this: depth 48.5 and, by the distance's rounding up (250 at most, where it is
    // subnormal) and the difference's rounding down (500), less than 800.  To the nearest, the distance became 0 at T < 2.1e-47.
    const float floor_l = fmaxf(__fsub_rd(top, __double2float_ru(48.5 / slope)), -3.402823466e38f);
    // of a finite logit, without branches, so that several run at once
    const auto biased = [&](float l) { return fixed_exp2_biased(top64 - static_cast<double>(fmaxf(l, floor_l)), slope16, sh.table); };
    const auto weight = [&](float l) { return static_cast<unsigned long long>(__double_as_longlong(biased(l))) - 0x4330000000000000ull; };
    // the first word whose sum exceeds u * all: at least this much
    const auto target_of = [&](unsigned long long all) {
        const double u = sh.u, at = u > 0.0 ? u * static_cast<double>(all) : 0.0;
        return (at < static_cast<double>(all) ? min(static_cast<unsigned long long>(at), all - 1) : all - 1) + 1;
    };

    // ---- few words
    const int groups = static_cast<int>(blockDim.x) / p.group;   // of a CTA
    if (!alone && k <= groups * ranks * 3 / 4) {
        const int n = groups * ranks;      // at most 256
        for (int i = t; i < n; i += blockDim.x) sh.all_groups[i] = *cluster.map_shared_rank(&sh.group_top[i % groups], i / groups);
        __syncthreads();
        // the rank of each: four lanes to a group
        for (int i = t >> 2; i < ((n + 7) & ~7); i += blockDim.x >> 2) {
            const float mine = i < n ? sh.all_groups[i] : 0.f;
            int before = 0;
            for (int j = t & 3; j < n; j += 4) {
                const float other = sh.all_groups[j];
                before += other > mine || (other == mine && j < i);
            }
            before += __shfl_xor_sync(0xFFFFFFFFu, before, 1);
            before += __shfl_xor_sync(0xFFFFFFFFu, before, 2);
            if (i < n && before == k - 1) sh.floor = mine;
        }
        __syncthreads();
        const float floor = sh.floor;
        each([&](int c, int j, const float (&v)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[i] >= floor && v[i] > -INFINITY) {
                    const uint32_t at = atomicAdd(&sh.candidates, 1u);
                    if (at < kCandidates) sh.candidate[at] = {v[i], row.word(c, j, lane, i)};
                }
        });
        cluster.sync();
        if (warp == 0) {
            const uint32_t end = warp_scan(lane < ranks ? *cluster.map_shared_rank(&sh.candidates, lane) : 0u, lane);
            if (lane < kMostCtas) sh.ends[lane] = end;
        }
        __syncthreads();
        const uint32_t all = sh.ends[kMostCtas - 1];
        if (all <= kCandidates) {
            if (rank == 0) {
                const int count = static_cast<int>(all);
                for (int i = t; i < count; i += blockDim.x) {
                    int r = 0;
                    while (i >= static_cast<int>(sh.ends[r])) ++r;
                    sh.few.all[i] = cluster.map_shared_rank(&sh, r)->candidate[i - static_cast<int>(r ? sh.ends[r - 1] : 0u)];
                }
                __syncthreads();
                // in their order, the first k
                for (int i = t; i < count; i += blockDim.x) {
                    const Candidate mine = sh.few.all[i];
                    int before = 0;
                    for (int j = 0; j < count; ++j) {
                        const Candidate other = sh.few.all[j];
                        before += other.l > mine.l || (other.l == mine.l && other.word < mine.word);
                    }
                    if (before < k) {
                        sh.few.kept[before] = mine;
                        sh.few.weight[before] = weight(mine.l);
                    }
                }
                __syncthreads();
                // the first of those by top_p and min_p: what stands before each of them, one to a thread
                const int first = static_cast<int>(k < count ? k : count);
                const double top_p = sh.top_p, deepest = sh.deepest;
                int kept = 0;
                for (int from = 0; from < first; from += blockDim.x) {
                    const int i = from + t;
                    unsigned long long whole = 0, before = 0;
#pragma unroll 4
                    for (int j = 0; j < first; ++j) {
                        const unsigned long long w = sh.few.weight[j];
                        whole += w;
                        before += j < i ? w : 0ull;
                    }
                    const double goal = top_p > 0.0 ? top_p * static_cast<double>(whole) : 0.0;
                    // (what is kept is a beginning of their order)
                    const bool keep = i < first && (i == 0 || ((!(top_p < 1.0) || static_cast<double>(before) < goal) && depth(sh.few.kept[i].l) <= deepest));
                    kept += __syncthreads_count(keep);
                }
                for (int i = t; i < kept; i += blockDim.x) {
                    const int word = sh.few.kept[i].word;
                    const unsigned long long own = sh.few.weight[i];
                    unsigned long long run = 0, sum = 0;
#pragma unroll 4
                    for (int j = 0; j < kept; ++j) {
                        const unsigned long long w = sh.few.weight[j];
                        sum += w;
                        run += sh.few.kept[j].word <= word ? w : 0ull;
                    }
                    const unsigned long long target = target_of(sum);
                    if (run >= target && run - own < target) {
                        p.tokens[m] = word;
                        if (p.probs) p.probs[m] = static_cast<float>(static_cast<double>(own) / static_cast<double>(sum));
                    }
                }
            }
            cluster.sync();                // nobody leaves while its candidates may still be read
            return;
        }
    }

    // ---- the kept words: above tau, and `quota` of those that equal it
    uint32_t tau = 0;                      // key; nothing that can be drawn is at 0
    uint32_t quota = 0, equal_all = 0;     // equal_all: words at tau
    // bins of equal width below the largest logit; falls with l, as every step of it does (halves: the difference of two finite numbers is
    // finite; the floor is read off a sum with 2^23)
    const auto bin_of = [&](float l, float scale) {
        const float d = fminf(fmaf(l, -0.5f, half_top) * (2.f * scale), static_cast<float>(kBins - 1));
        return static_cast<int>(__float_as_uint(__fadd_rd(d, 8388608.f)) & (kBins - 1));
    };
    const auto at_least = [](uint32_t key) { return key ? of_key(key) : -3.402823466e38f; };       // keys from `key` on that are no -inf
    // f(bin of this lane, span) in the first CTA: a warp takes 32 bins at a time
    const auto spans = [&](auto&& f) {
        for (int span = warp; span < kSpans; span += warps) f(span * 32 + lane, span);
    };
    // The histograms of the cluster's CTAs, joined in the first one's own.
    const auto join = [&](bool by_weight) {
        for (int i = t; i < kBins; i += blockDim.x) {
            uint32_t n[kMostCtas];
            unsigned long long w[kMostCtas] = {};
#pragma unroll
            for (int r = 0; r < kMostCtas; ++r) n[r] = r < ranks ? *cluster.map_shared_rank(&sh.count[i], r) : 0u;
            if (by_weight)
#pragma unroll
                for (int r = 0; r < kMostCtas; ++r) w[r] = r < ranks ? *cluster.map_shared_rank(&sh.weight[i], r) : 0ull;
#pragma unroll
            for (int r = 1; r < kMostCtas; ++r) { n[0] += n[r]; w[0] += w[r]; }
            sh.count[i] = n[0];
            sh.weight[i] = w[0];
        }
        __syncthreads();
    };
    // The first bin of the first CTA's histogram at which `reached` holds of the sums from the first bin on and what stands above them: to sh.found
    // (first, above_count, above, active: the words in it).  For all its threads.
    const auto find = [&](bool by_weight, auto&& reached) {
        spans([&](int b, int span) {
            if (by_weight) {
                const unsigned long long w = warp_add(sh.weight[b]);
                if (lane == 0) sh.span_weight[span] = w;
            } else {
                const uint32_t n = __reduce_add_sync(0xFFFFFFFFu, sh.count[b]);
                if (lane == 0) sh.span_count[span] = n;
            }
        });
        __syncthreads();
        if (warp == 0) {                   // to the sums before each span
            if (by_weight) {
                const unsigned long long own = sh.span_weight[lane];
                sh.span_weight[lane] = sh.found.above + warp_scan(own, lane) - own;
            } else {
                const uint32_t own = sh.span_count[lane];
                sh.span_count[lane] = sh.found.above_count + warp_scan(own, lane) - own;
            }
            if (lane == 0) sh.found.first = -1;
        }
        __syncthreads();
        spans([&](int b, int span) {
            const uint32_t own = sh.count[b];
            const unsigned long long own_weight = sh.weight[b];
            uint32_t n = 0;
            unsigned long long w = 0;
            if (by_weight) w = sh.span_weight[span] + warp_scan(own_weight, lane);
            else n = sh.span_count[span] + warp_scan(own, lane);
            // sums do not fall, so that one bin is the first
            if (reached(n, w) && !(b > 0 && reached(n - own, w - own_weight))) {
                sh.found.first = b;
                sh.found.active = own;
                sh.found.above_count = n - own;
                sh.found.above = w - own_weight;
            }
        });
        __syncthreads();
    };
    // Behind the first CTA's search: what it found comes into every CTA's own sh.found.  (It is written next behind another
    // cluster.sync.)  The histograms and the lists of words have been read, and are emptied.
    const auto publish = [&] {
        cluster.sync();
        if (rank > 0 && warp == 0)
            for (int i = lane; i < static_cast<int>(sizeof(Found) / 4); i += 32)
                reinterpret_cast<uint32_t*>(&sh.found)[i] = *cluster.map_shared_rank(reinterpret_cast<uint32_t*>(&sh.found) + i, 0);
        for (int i = t; i < kBins; i += blockDim.x) {
            sh.count[i] = 0;
            sh.weight[i] = 0;
        }
        if (t == 0) { sh.listed = sh.candidates; sh.candidates = 0; }
        __syncthreads();
    };
    const auto width_of = [](uint32_t keys) {                    // a bin holds 2^width keys
        int width = 0;
        while ((keys >> width) >= kBins) ++width;
        return width;
    };
    // The first number, from the largest logit down, at which the sum over the words of keys >= `least` reaches its goal, when it is known to lie in
    // the bins sh.found.first .. last of width 1 / scale, with sh.found.active words.  Sets tau and equal_all.
    // Weights: every word's weight is made here, once, and added up, of all and of those above those bins; all less `excess`, times top_p, is the goal.
    bool listed = false;                   // the words in the bins are in the CTAs' lists, the weight above them in sh.warp_beyond
    const auto narrow = [&](bool by_weight, auto&& reached, uint32_t least, float scale, unsigned long long excess) {
        const int first = sh.found.first, last = sh.found.last;
        // keys of the bins' words: their ends, and more than the roundings of bin_of and of the ends can be
        uint32_t low = 0, high = key_of(top);
        if (scale > 1e-30f && scale < 1e30f) {
            const float up = static_cast<float>(first) / scale, down = static_cast<float>(last + 1) / scale;
            const float slack = (fabsf(top) + down) * 0x1p-21f;
            if (first > 0) high = key_of(canonical(fminf(top, top - up + slack)));
            if (last < kBins - 1) low = key_of(canonical(top - down - slack));
        }
        bool begin = by_weight;            // the weights are still to be added up
        while (true) {
            const bool few = sh.found.active <= kWords;          // enough for the first CTA
            const int width = width_of(high - low);
            // (a thread's sums are below 2^53: 2^50 at most)
            // words below `least` count for nothing; -inf weighs nothing by itself, but where even the lowest number weighs something
            const bool masked = least != 0 || floor_l == -3.402823466e38f;
            double beyond64 = 0.0, whole64 = 0.0;
            const float high_l = of_key(high), least_l = at_least(least), low_l = fmaxf(least_l, low > 0x007FFFFFu ? of_key(low) : -INFINITY);
            each([&](int c, int j, const float (&v)[4]) {
                double w[4] = {};
                if (begin) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = biased(v[i]) - kRound[1];
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = v[i] >= least_l ? w[i] : 0.0;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        whole64 += w[i];
                        // without its upper half a number is as good as 0
                        beyond64 += __hiloint2double(v[i] > high_l ? __double2hiint(w[i]) : 0, __double2loint(w[i]));
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (v[i] <= high_l && v[i] >= low_l) {
                        const int b = bin_of(v[i], scale);
                        if (b < first) {
                            beyond64 += w[i];
                        } else if (b <= last) {
                            if (few) {
                                const uint32_t at = atomicAdd(&sh.candidates, 1u);
                                if (at < kWords) sh.active[at] = {v[i], row.word(c, j, lane, i)};
                            } else {
                                const int at = static_cast<int>((high - key_of(v[i])) >> width);
                                atomicAdd(&sh.count[at], 1u);
                                if (by_weight) atomicAdd(&sh.weight[at], weight(v[i]));
                            }
                        }
                    }
                }
            });
            if (begin) {
                unsigned long long beyond = warp_add(static_cast<unsigned long long>(beyond64)), whole = warp_add(static_cast<unsigned long long>(whole64));
                if (lane == 0) {
                    sh.warp_beyond[warp] = beyond;
                    sh.warp_total[warp] = whole;
                }
                __syncthreads();
                if (warp == 0) {
                    beyond = warp_add(lane < warps ? sh.warp_beyond[lane] : 0ull);
                    whole = warp_add(lane < warps ? sh.warp_total[lane] : 0ull);
                    if (lane == 0) { sh.beyond = beyond; sh.whole = whole; }
                }
                listed = few;
            }
            cluster.sync();
            if (rank == 0) {
                int n = 0;
                if (!few) {
                    join(by_weight);
                } else {
                    // the words into this CTA's own memory
                    if (warp == 0) {
                        const uint32_t own = lane < ranks ? min(*cluster.map_shared_rank(&sh.candidates, lane), static_cast<uint32_t>(kWords)) : 0u;
                        const uint32_t end = warp_scan(own, lane);
                        if (lane < kMostCtas) sh.ends[lane] = end;
                    }
                    __syncthreads();
                    n = static_cast<int>(min(sh.ends[kMostCtas - 1], static_cast<uint32_t>(kWords)));
                    for (int i = t; i < n; i += blockDim.x) {
                        int r = 0;
                        while (i >= static_cast<int>(sh.ends[r])) ++r;
                        sh.words[i] = cluster.map_shared_rank(&sh, r)->active[i - static_cast<int>(r ? sh.ends[r - 1] : 0u)].l;
                    }
                    __syncthreads();
                }
                if (begin) {
                    if (warp == 0) {
                        const unsigned long long up = cluster_sum(cluster, ranks, &sh.beyond, lane), all = cluster_sum(cluster, ranks, &sh.whole, lane);
                        if (lane == 0) {
                            sh.found.above += up;
                            sh.found.goal = fmax(sh.top_p > 0.0 ? sh.top_p * static_cast<double>(all - excess) : 0.0, 0.5);       // one word at least
                        }
                    }
                    __syncthreads();
                }
                if (!few) {
                    find(by_weight, reached);
                    if (t == 0) {
                        sh.found.done = width == 0;
                        sh.found.tau = high - static_cast<uint32_t>(sh.found.first);
                        sh.found.equal = sh.found.active;
                    }
                } else {
                    // the same search among the words
                    uint32_t from = low, to = high;
                    while (true) {
                        const int w = width_of(to - from);
                        for (int i = t; i < n; i += blockDim.x) {
                            const uint32_t key = key_of(sh.words[i]);
                            if (key < from || key > to) continue;
                            const int at = static_cast<int>((to - key) >> w);
                            atomicAdd(&sh.count[at], 1u);
                            if (by_weight) atomicAdd(&sh.weight[at], weight(sh.words[i]));
                        }
                        __syncthreads();
                        find(by_weight, reached);
                        const int bin = sh.found.first;
                        if (w == 0 || bin < 0) {
                            if (t == 0) {
                                sh.found.done = 1;
                                sh.found.tau = to - static_cast<uint32_t>(bin);
                                sh.found.equal = sh.found.active;
                            }
                            break;
                        }
                        if (sh.found.active <= 32) {
                            // the words of that bin, to a lane of one warp each
                            const uint32_t last_key = to - (static_cast<uint32_t>(bin) << w), first_key = last_key - ((1u << w) - 1u);
                            if (t == 0) sh.joined = 0;
                            __syncthreads();
                            for (int i = t; i < n; i += blockDim.x) {
                                const uint32_t key = key_of(sh.words[i]);
                                if (key <= last_key && key >= first_key && key >= from) sh.lanes[atomicAdd(&sh.joined, 1u) & 31u] = sh.words[i];
                            }
                            __syncthreads();
                            if (warp == 0) {
                                const int count = static_cast<int>(min(sh.joined, 32u));
                                const float l = lane < count ? sh.lanes[lane] : -INFINITY;
                                const unsigned long long own = by_weight && lane < count ? weight(l) : 0ull;
                                uint32_t above_n = sh.found.above_count, equal = 0;
                                unsigned long long above_w = sh.found.above;
                                for (int j = 0; j < count; ++j) {
                                    const float other = __shfl_sync(0xFFFFFFFFu, l, j);
                                    const unsigned long long its = __shfl_sync(0xFFFFFFFFu, own, j);
                                    above_n += other > l;
                                    above_w += other > l ? its : 0ull;
                                    equal += other == l;
                                }
                                const bool here = lane < count && reached(above_n + equal, above_w + equal * own) && !reached(above_n, above_w);
                                const unsigned lanes_here = __ballot_sync(0xFFFFFFFFu, here);          // of one number
                                if (lane == __ffs(lanes_here) - 1) {
                                    sh.found.done = 1;
                                    sh.found.tau = key_of(l);
                                    sh.found.equal = equal;
                                    sh.found.above_count = above_n;
                                    sh.found.above = above_w;
                                }
                            }
                            break;
                        }
                        for (int i = t; i < kBins; i += blockDim.x) {
                            sh.count[i] = 0;
                            sh.weight[i] = 0;
                        }
                        to -= static_cast<uint32_t>(bin) << w;
                        const uint32_t span = (1u << w) - 1u;
                        if (to - from > span) from = to - span;
                        __syncthreads();
                    }
                }
            }
            publish();
            begin = false;
            const int bin = sh.found.first;
            const bool done = sh.found.done;
            if (bin < 0) return false;
            if (done) {
                tau = sh.found.tau;
                equal_all = quota = sh.found.equal;
                return true;
            }
            high -= static_cast<uint32_t>(bin) << width;
            const uint32_t span = (1u << width) - 1u;
            if (high - low > span) low = high - span;
        }
    };
    const auto count_bins = [&](float scale) {
        each([&](int, int, const float (&v)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[i] > -INFINITY) atomicAdd(&sh.count[bin_of(v[i], scale)], 1u);
        });
    };

    if (k < p.V) {
        const auto reached = [&](uint32_t n, unsigned long long) { return n >= static_cast<uint64_t>(k); };
        count_bins(kBinsPerUnit);
        cluster.sync();
        if (rank == 0) {
            if (t == 0) { sh.found.above_count = 0; sh.found.above = 0; sh.found.done = 0; }
            join(false);
            find(false, reached);
            if (t == 0) sh.found.last = sh.found.first;
        }
        publish();
        if (sh.found.first >= 0 && narrow(false, reached, 0, kBinsPerUnit, 0)) quota = static_cast<uint32_t>(k - sh.found.above_count);
        __syncthreads();
    }
    // top-p: among the words from tau on
    const bool by_p = sh.top_p < 1.0;
    unsigned long long mine = 0;
    if (by_p) {
        const uint32_t tau_k = tau, quota_k = quota, equal_k = equal_all;
        const float scale = fminf(static_cast<float>(slope * kBinsPerUnit), 1e30f), least_l = at_least(tau_k);
        // their weight, about, and how many there are in bins of depth
        double sum = 0.0;
        each([&](int, int, const float (&v)[4]) {
            float some = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = v[i] >= least_l;
                float w;
                asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(fmaf(v[i], -0.5f, half_top) * (-2.f * slope_f)));
                some += in ? w : 0.f;
                if (in) atomicAdd(&sh.count[bin_of(v[i], scale)], 1u);
            }
            sum += static_cast<double>(some);
        });
        const double about = warp_add(sum);
        if (lane == 0) sh.warp_real[warp] = about;
        __syncthreads();
        if (warp == 0) {
            const double all = warp_add(lane < warps ? sh.warp_real[lane] : 0.0);
            if (lane == 0) sh.real = all;
        }
        const unsigned long long at_tau = tau_k ? weight(of_key(tau_k)) : 0ull, excess = (equal_k - quota_k) * at_tau;
        cluster.sync();
        if (rank == 0) {
            if (warp == 0) {
                const double sum_all = cluster_sum(cluster, ranks, &sh.real, lane);
                if (lane == 0) { sh.real = sum_all; sh.found.above_count = 0; sh.found.above = 0; sh.found.done = 0; }
            }
            join(false);
            // What the words of bin b weigh together, in units of 2^S: their count times what its ends weigh, a little more or less for
            // bin_of's roundings and the weights' own.  The sum of all is within 1.5e-5 of what was added up (a product of y <= 47 is
            // off by 3 * 2^-24 of it, and its power by as much times y ln 2) and of the weights' own roundings, half a unit each (2^-29 of the largest
            // weight in all at 2^17 words, 2^-13 at 2^25, 1/8 at 2^30); the sums of a thousand terms here within 1e-6 of all.  Where the scale has
            // left its range, the bins say nothing, and all words are looked at.
            const float unit = exp2f(static_cast<float>(-p.shift)), roundings = 0.5f * unit * static_cast<float>(p.V);
            const float all = static_cast<float>(sh.real), cut = static_cast<float>(static_cast<double>(excess) / static_cast<double>(1ull << p.shift));
            const float low_all = all * (1.f - 1.5e-5f) - roundings, high_all = all * (1.f + 1.5e-5f) + roundings, top_p = static_cast<float>(sh.top_p);
            const float low_goal = top_p * fmaxf(low_all - cut, 0.f) * (1.f - 1e-6f), high_goal = top_p * fmaxf(high_all - cut, 0.f) * (1.f + 1e-6f);
            const bool known = scale > 1e-30f && scale < 1e30f;
            const auto most_of = [&](int b) { return static_cast<float>(sh.count[b]) * (exp2f(static_cast<float>(b) / -kBinsPerUnit) * (1.f + 2e-5f) + unit); };
            const auto least_of = [&](int b) {
                return b == kBins - 1 ? 0.f : static_cast<float>(sh.count[b]) * fmaxf(exp2f(static_cast<float>(b + 1) / -kBinsPerUnit) * (1.f - 2e-5f) - unit, 0.f);
            };
            spans([&](int b, int span) {
                const float most = warp_add(most_of(b)), least = warp_add(least_of(b));
                if (lane == 0) { sh.span_most[span] = most; sh.span_least[span] = least; }
            });
            __syncthreads();
            if (warp == 0) {               // to the sums before each span
                const float most = sh.span_most[lane], least = sh.span_least[lane], most_to = warp_scan(most, lane), least_to = warp_scan(least, lane);
                sh.span_most[lane] = most_to - most;
                sh.span_least[lane] = least_to - least;
                if (lane == 31) { sh.most = most_to; sh.least = least_to; }
                if (lane == 0) { sh.found.first = known ? kBins - 1 : 0; sh.found.last = kBins - 1; sh.found.active = 0; }
            }
            __syncthreads();
            if (known)
                spans([&](int b, int span) {
                    // the sum up to bin b, from above and as all but what is below it: may it, and must it have reached the goal?
                    const float most = sh.span_most[span] + warp_scan(most_of(b), lane), least = sh.span_least[span] + warp_scan(least_of(b), lane);
                    const float slack = 3e-6f * sh.most;
                    const float up = fminf(most, high_all - (sh.least - least)) + slack, down = fmaxf(least, low_all - (sh.most - most)) - slack;
                    const uint32_t may = __reduce_min_sync(0xFFFFFFFFu, static_cast<uint32_t>(up >= low_goal ? b : kBins));
                    const uint32_t must = __reduce_min_sync(0xFFFFFFFFu, static_cast<uint32_t>(down >= high_goal ? b : kBins));
                    if (lane == 0 && may < kBins) atomicMin(&sh.found.first, static_cast<int>(may));
                    if (lane == 0 && must < kBins) atomicMin(&sh.found.last, static_cast<int>(must));
                });
            __syncthreads();
            spans([&](int b, int) {
                const uint32_t n = __reduce_add_sync(0xFFFFFFFFu, b >= sh.found.first && b <= sh.found.last ? sh.count[b] : 0u);
                if (lane == 0 && n) atomicAdd(&sh.found.active, n);
            });
        }
        publish();
        // (all words' sum reaches the goal, so that there is a border)
        if (narrow(true, [&](uint32_t, unsigned long long w) { return static_cast<double>(w) >= sh.found.goal; }, tau_k, scale, excess)) {
            const double goal = sh.found.goal;
            // of the words at tau, those before which the weight is below the goal
            const double before = static_cast<double>(sh.found.above), each_one = static_cast<double>(weight(of_key(tau)));
            const double n = goal > before ? ceil((goal - before) / each_one) : 0.0;
            quota = n < 1.0 ? 1u : n < static_cast<double>(equal_all) ? static_cast<uint32_t>(n) : equal_all;
            if (tau == tau_k && quota > quota_k) quota = quota_k;
        }
    }

    // ---- the draw
    // words at tau before this warp's, where not all are kept
    const bool ranked = quota < equal_all;
    uint32_t equals_before = 0;
    if (ranked) {
        uint32_t n = 0;
        each([&](int, int, const float (&v)[4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) n += key_of(v[i]) == tau;
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
        if (warp == 0) {
            n = cluster_sum(cluster, rank, &sh.equal, lane);
            if (lane == 0) sh.joined = n;
        }
        __syncthreads();
        equals_before = sh.joined;
        equals_before += sh.warp_equal[warp];
    }
    // f(chunk, vector, weights of its elements) over this lane's vectors in the words' order, weight 0 for what is not kept.
    const bool by_depth = sh.deepest < INFINITY;
    const auto walk = [&](auto&& f) {
        uint32_t before = equals_before;
        each([&](int c, int j, const float (&v)[4]) {
            uint32_t rank_here = 0;
            if (ranked) {
                uint32_t n = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) n += key_of(v[e]) == tau;
                if (__any_sync(0xFFFFFFFFu, n > 0)) {
                    const uint32_t to = warp_scan(n, lane);
                    rank_here = before + to - n;
                    before += __shfl_sync(0xFFFFFFFFu, to, 31);
                }
            }
            unsigned long long w[4] = {};
            bool in[4], some = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t key = key_of(v[e]);
                in[e] = key > tau;
                if (key == tau) in[e] = !ranked || rank_here++ < quota;
                in[e] = in[e] && v[e] > -INFINITY;
                if (by_depth && in[e]) in[e] = depth(v[e]) <= sh.deepest;
                some = some || in[e];
            }
            if (__any_sync(0xFFFFFFFFu, some)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = weight(v[e]);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = in[e] ? w[e] : 0ull;
            }
            f(c, j, w);
        });
    };
    mine = 0;
    if (by_p && listed && !by_depth && !ranked) {
        // what lies above the bins that top-p's border was looked for in has been added up there; those in them are listed
        if (lane == 0) sh.warp_total[warp] = sh.warp_beyond[warp];
        __syncthreads();
        const int per_warp = p.chunks * p.vectors * 128, base = row.first - warp * per_warp;
        for (int i = t; i < static_cast<int>(sh.listed); i += blockDim.x) {
            const Candidate one = sh.active[i];
            if (key_of(one.l) >= tau) atomicAdd(&sh.warp_total[(one.word - base) / per_warp], weight(one.l));
        }
        __syncthreads();
        mine = sh.warp_total[warp];
        __syncthreads();                   // sh.warp_total is written again
    } else {
        walk([&](int, int, const unsigned long long (&w)[4]) { mine += w[0] + w[1] + (w[2] + w[3]); });
        mine = warp_add(mine);
    }
    if (lane == 0) sh.warp_total[warp] = mine;
    __syncthreads();
    if (warp == 0) {
        const unsigned long long own = lane < warps ? sh.warp_total[lane] : 0ull, to = warp_scan(own, lane);
        if (lane < warps) sh.warp_total[lane] = to - own;
        if (lane == 31) sh.total = to;
    }
    cluster.sync();
    if (warp == 0) {
        const unsigned long long own = lane < ranks ? *cluster.map_shared_rank(&sh.total, lane) : 0ull;
        const unsigned long long before = warp_add(lane < rank ? own : 0ull), sum = warp_add(own);
        if (lane == 0) { sh.base = before; sh.all = sum; }
    }
    __syncthreads();
    const unsigned long long all = sh.all;
    unsigned long long base = sh.base;
    base += sh.warp_total[warp];
    const unsigned long long target = target_of(all);
    if (base < target && target <= base + mine) {                // this warp has it
        unsigned long long before = base;
        bool done = false;
        walk([&](int c, int j, const unsigned long long (&w)[4]) {
            const unsigned long long own = w[0] + w[1] + (w[2] + w[3]);
            const unsigned long long to = warp_scan(own, lane) + before;
            before = __shfl_sync(0xFFFFFFFFu, to, 31);
            if (!done && to >= target && to - own < target) {
                unsigned long long run = to - own, its = 0;
                int word = -1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    run += w[e];
                    if (word < 0 && run >= target) { word = e; its = w[e]; }
                }
                p.tokens[m] = row.word(c, j, lane, word);
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
    // a row may start inside a vector
    const bool aligned = atb::aligned16(p.logits) && (p.M == 1 || p.ld * static_cast<int64_t>(sizeof(T)) % 16 == 0);
    const int64_t positions = p.V + (aligned ? 0 : 16 / static_cast<int64_t>(sizeof(T)) - 1);
    // CTAs per row: what its words need, and more, of 1024 words at least, while the rows leave SMs idle.  Vectors per thread: as many as there
    // are where the SMs are full (what a warp does once per pass counts for more words), else as few as fill the threads.
    int ctas = 1;
    while (ctas < kMostCtas && (positions > static_cast<int64_t>(ctas) * kMostThreads * kPerThread || (p.M * ctas * 2 <= atb::kSmCount && positions >= ctas * 2 * 1024))) ctas *= 2;
    const int64_t share = atb::ceil_div(positions, ctas);
    p.vectors = kVectors;
    if (p.M * ctas <= atb::kSmCount)
        while (p.vectors > 2 && share <= static_cast<int64_t>(kMostThreads) * 4 * (p.vectors / 2)) p.vectors /= 2;
    const int64_t threads = atb::ceil_div(share, 4 * p.vectors);
    p.chunks = static_cast<int>(atb::ceil_div(threads, kMostThreads));
    int block = static_cast<int>(atb::round_up(atb::ceil_div(threads, p.chunks), 32));
    if (block < 64) block = 64;
    p.group = 1;                           // 256 groups at most, in all
    while (block / p.group * ctas > kMostGroups) p.group *= 2;
    int log2v = 0;
    while ((1ll << log2v) < p.V) ++log2v;
    p.shift = 62 - log2v < 45 ? 62 - log2v : 45;
    const unsigned grid = static_cast<unsigned>(p.M * ctas);
    const size_t smem = static_cast<size_t>(block) * p.vectors * sizeof(float4);
    constexpr size_t most = static_cast<size_t>(kMostThreads) * kPerThread * sizeof(float);
    const cudaError_t e = p.chunks == 1 ? atb::allow_shared_memory<&sample_kernel<T, true>>(most) : atb::allow_shared_memory<&sample_kernel<T, false>>(most);
    if (e != cudaSuccess) return e;
    auto kernel = p.chunks == 1 ? sample_kernel<T, true> : sample_kernel<T, false>;
    return atb::launch_dependent(kernel, grid, static_cast<unsigned>(block), static_cast<unsigned>(ctas), smem, st, p);
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
