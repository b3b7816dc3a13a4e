// Residual norm, backward (sm_100a).  With n = norm(h), g = dz w, and t the whole gradient that arrives at h:
//
//   t = dh + r (g - sum(g) / N - n sum(g n) / N)          (rms: without the sum of g)
//   dx = scale t,  du = gate t,  df = du, or with a norm of f, q = du pw and m = norm(f):  r_f (q - sum(q) / N - m sum(q m) / N)
//   over the rows: S0 = sum dz n, S1 = sum dz, S2 = sum t m (sum t f without a norm of f), S3 = sum t
//   dw = S0, db = S1, dgate = pw S2 + pb S3 (S2), dpw = gate S2, dpb = gate S3
//
// Bound by memory: dz, dh, x and f are read, dx and df written, once.  h is made of x and f again, unrounded: its rounding to bf16 would
// be in dw (2^-9 of every term, where dw itself may be FP32).  Blocks stay and walk the rows, so that the sums over the rows stay in
// registers; a thread has 8 columns (16 where rows are wider than 4096), the row is read from shared memory once for the sums of
// g and again for what follows them, and the next rows are on their way (cp.async) meanwhile.  Walkers leave their sums in the
// workspace; another kernel adds those up in a fixed order.
#include "atb_residual_norm.cuh"

namespace residual_norm {
namespace {

constexpr int kBlockThreads = 512;         // per SM, 128 registers each
// Two FP32 rows of more than 4096 elements leave no room for dh beside x, f and dz twice: it is loaded where it is used.
template <class TX, class TF, int VEC, int NV>
constexpr bool kDirect = sizeof(TX) + sizeof(TF) == 8 && NV * VEC > 8;
template <class TX, class TF, int VEC, int TPR, int NV>
constexpr int kStage = static_cast<int>((kDirect<TX, TF, VEC, NV> ? 1 : 2) * RowSource<TX, VEC, TPR, NV>::STAGE_BYTES + 2 * RowSource<TF, VEC, TPR, NV>::STAGE_BYTES);
__host__ __device__ constexpr int blocks_of(int tpr) { return kBlockThreads / (tpr == 32 ? 128 : tpr); }
template <class TX, class TF, int VEC, int TPR, int NV>
__host__ __device__ constexpr int ahead_of() {
    const int stages = 208 * 1024 / (blocks_of(TPR) * kStage<TX, TF, VEC, TPR, NV>);
    return stages > 4 ? 3 : stages - 1;
}

template <class TX, class TF, int VEC, int TPR, int NV, bool POST>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, blocks_of(TPR)) residual_norm_backward_kernel(const BwdParams p) {
    using SX = RowSource<TX, VEC, TPR, NV>;
    using SF = RowSource<TF, VEC, TPR, NV>;
    using Shared = std::conditional_t<SX::SHARED, SX, SF>;
    constexpr bool DIRECT = kDirect<TX, TF, VEC, NV>;
    constexpr int WALKERS = TPR == 32 ? 4 : 1, W = TPR / 32, AHEAD = ahead_of<TX, TF, VEC, TPR, NV>(), STAGES = AHEAD + 1;
    static_assert(AHEAD >= 1, "shared memory");
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float red[2][2][W][2];
    const int t = TPR == 32 ? threadIdx.x & 31 : threadIdx.x;
    const int N = static_cast<int>(p.N), col = t * VEC;                 // group i: columns col + i TPR VEC ..
    const int64_t first = static_cast<int64_t>(blockIdx.x) * WALKERS + (TPR == 32 ? threadIdx.x >> 5 : 0), step = static_cast<int64_t>(gridDim.x) * WALKERS;
    const uint32_t base = sm100::smem_u32(ring);
    const SF sf(base, p.f, p.ldf, p.M, N, t), sdz(base + STAGES * SF::STAGE_BYTES, p.dz, p.lddz, p.M, N, t);
    const SX sx(base + 2 * STAGES * SF::STAGE_BYTES, p.x, p.ldx, p.M, N, t), sdh(base + STAGES * (2 * SF::STAGE_BYTES + SX::STAGE_BYTES), p.dh, p.lddh, p.M, N, t);
    const float inv_n = 1.f / static_cast<float>(N);
    const bool has_dh = p.dh != nullptr;
    const auto fetch = [&](int stage, int64_t m) {
        sx.fetch(stage, m);
        sf.fetch(stage, m);
        sdz.fetch(stage, m);
        if constexpr (!DIRECT)
            if (has_dh) sdh.fetch(stage, m);
    };
    sm100::grid_dependency_wait();
    sm100::grid_dependency_launch();
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) {
        if (first + s * step < p.M) fetch(s, first + s * step);
        async_commit();
    }
    float s0[NV][VEC] = {}, s1[NV][VEC] = {}, s2[NV][VEC] = {}, s3[POST ? NV : 1][VEC] = {};
    int stage = 0, turn = 0;
    float mu = 0.f, r = 0.f, fmu = 0.f, fr = 0.f;
    const auto stats = [&](int64_t m, float& a, float& b, float& c, float& d) {
        if (m >= p.M) return;
        a = p.stats[m];
        b = p.stats[p.M + m];
        if constexpr (POST) { c = p.stats[2 * p.M + m]; d = p.stats[3 * p.M + m]; }
    };
    stats(first, mu, r, fmu, fr);
    for (int64_t m = first; m < p.M; m += step, turn ^= 1) {
        const int ahead = stage == 0 ? AHEAD : stage - 1;               // the stage that the row before this one has left
        if (m + AHEAD * step < p.M) fetch(ahead, m + AHEAD * step);
        async_commit();
        float next[4] = {};
        stats(m + step, next[0], next[1], next[2], next[3]);
        Raw<TX, VEC> direct[DIRECT ? NV : 1];
        if constexpr (DIRECT)
            if (has_dh)
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (col + i * TPR * VEC < N) load_raw<TX, VEC>(static_cast<const TX*>(p.dh) + m * p.lddh + col + i * TPR * VEC, direct[i]);
        async_wait<AHEAD>();
        row_barrier<Shared, VEC, TPR>();
        // f, or norm(f), and norm(h) of group i
        const auto values = [&](int i, float (&f)[VEC], float (&h)[VEC]) {
            const int n = col + i * TPR * VEC;
            float a[VEC], b[VEC];
            Raw<TF, VEC> rf;
            Raw<TX, VEC> rx;
            sf.read(stage, m, i, rf);
            to_float(rf, f);
            sx.read(stage, m, i, rx);
            if constexpr (POST) {
                weights<VEC>(p.v.pw, p.v.w32, n, 1.f, a);
                weights<VEC>(p.v.pb, p.v.w32, n, 0.f, b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    f[e] = (f[e] - fmu) * fr;
                    h[e] = fmaf(f[e], a[e], b[e]);
                }
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) h[e] = f[e];
            }
            to_float(rx, b);
            weights<VEC>(p.v.gate, p.v.w32, n, 1.f, a);
#pragma unroll
            for (int e = 0; e < VEC; ++e) h[e] = (fmaf(p.scale, b[e], a[e] * h[e]) - mu) * r;
        };
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (col + i * TPR * VEC < N) {
                float f[VEC], h[VEC], dz[VEC], w[VEC];
                values(i, f, h);
                Raw<TF, VEC> raw;
                sdz.read(stage, m, i, raw);
                to_float(raw, dz);
                weights<VEC>(p.v.w, p.v.w32, col + i * TPR * VEC, 1.f, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    s0[i][e] = fmaf(dz[e], h[e], s0[i][e]);
                    s1[i][e] += dz[e];
                    const float g = dz[e] * w[e];
                    s[0] += g;
                    s[1] = fmaf(g, h[e], s[1]);
                }
            }
        row_sum<TPR, 2>(s, red[0][turn]);
        const float m0 = p.center ? s[0] * inv_n : 0.f, m1 = s[1] * inv_n;
        float q[POST ? NV : 1][VEC], k[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (col + i * TPR * VEC < N) {
                const int n = col + i * TPR * VEC;
                float f[VEC], h[VEC], dz[VEC], w[VEC];
                values(i, f, h);
                Raw<TF, VEC> raw;
                sdz.read(stage, m, i, raw);
                to_float(raw, dz);
                weights<VEC>(p.v.w, p.v.w32, n, 1.f, w);
                // dz becomes t
#pragma unroll
                for (int e = 0; e < VEC; ++e) dz[e] = r * (fmaf(dz[e], w[e], -m0) - h[e] * m1);
                if (has_dh) {
                    if constexpr (DIRECT) {
                        to_float(direct[i], w);
                    } else {
                        Raw<TX, VEC> rx;
                        sdh.read(stage, m, i, rx);
                        to_float(rx, w);
                    }
#pragma unroll
                    for (int e = 0; e < VEC; ++e) dz[e] += w[e];
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    s2[i][e] = fmaf(dz[e], f[e], s2[i][e]);
                    if constexpr (POST) s3[i][e] += dz[e];
                    w[e] = p.scale * dz[e];
                }
                if (p.dx) store_f<TX, VEC>(static_cast<TX*>(p.dx) + m * p.lddx + n, w);
                weights<VEC>(p.v.gate, p.v.w32, n, 1.f, w);
                if constexpr (POST) {
                    float pw[VEC];
                    weights<VEC>(p.v.pw, p.v.w32, n, 1.f, pw);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        q[i][e] = dz[e] * w[e] * pw[e];
                        k[0] += q[i][e];
                        k[1] = fmaf(q[i][e], f[e], k[1]);
                    }
                } else if (p.df) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) w[e] *= dz[e];
                    store_f<TF, VEC>(static_cast<TF*>(p.df) + m * p.lddf + n, w);
                }
            }
        if constexpr (POST) {
            row_sum<TPR, 2>(k, red[1][turn]);
            const float c0 = p.center ? -k[0] * inv_n : 0.f, c1 = -k[1] * inv_n;
            if (p.df)
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    if (col + i * TPR * VEC < N) {
                        Raw<TF, VEC> raw;
                        float f[VEC];
                        sf.read(stage, m, i, raw);
                        to_float(raw, f);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) f[e] = fr * fmaf((f[e] - fmu) * fr, c1, q[i][e] + c0);
                        store_f<TF, VEC>(static_cast<TF*>(p.df) + m * p.lddf + col + i * TPR * VEC, f);
                    }
        }
        // the row's stage is the next to be filled, by other threads than those that have just read it
        row_barrier<Shared, VEC, TPR>();
        mu = next[0]; r = next[1]; fmu = next[2]; fr = next[3];
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    if (p.part) {                          // a walker's sums: [walker][sums][N]
        float* out = p.part + first * (POST ? 4 : 3) * p.N;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int n = col + i * TPR * VEC;
            if (n < N) {
                store_f<float, VEC>(out + n, s0[i]);
                store_f<float, VEC>(out + p.N + n, s1[i]);
                store_f<float, VEC>(out + 2 * p.N + n, s2[i]);
                if constexpr (POST) store_f<float, VEC>(out + 3 * p.N + n, s3[i]);
            }
        }
    }
}

// ---------------------------------------------------------------------------------- any width
// One element's f (or norm(f)) and norm(h).
template <class TX, class TF, bool POST>
struct Element {
    const BwdParams& p;
    int64_t m;
    float mu, r, fmu, fr;
    __device__ __forceinline__ Element(const BwdParams& p_, int64_t m_) : p(p_), m(m_), mu(p_.stats[m_]), r(p_.stats[p_.M + m_]), fmu(0.f), fr(1.f) {
        if constexpr (POST) { fmu = p.stats[2 * p.M + m]; fr = p.stats[3 * p.M + m]; }
    }
    static __device__ __forceinline__ float weight(const void* w, int w32, int64_t n, float none) {
        float v[1];
        weights<1>(w, w32, static_cast<int>(n), none, v);
        return v[0];
    }
    __device__ __forceinline__ void operator()(int64_t n, float& f, float& h, float& dz) const {
        float v[1];
        load_f<TF, 1>(static_cast<const TF*>(p.f) + m * p.ldf + n, v);
        f = v[0];
        h = f;
        if constexpr (POST) {
            f = (f - fmu) * fr;
            h = fmaf(f, weight(p.v.pw, p.v.w32, n, 1.f), weight(p.v.pb, p.v.w32, n, 0.f));
        }
        load_f<TX, 1>(static_cast<const TX*>(p.x) + m * p.ldx + n, v);
        h = (fmaf(p.scale, v[0], weight(p.v.gate, p.v.w32, n, 1.f) * h) - mu) * r;
        load_f<TF, 1>(static_cast<const TF*>(p.dz) + m * p.lddz + n, v);
        dz = v[0];
    }
    // t from the means of g and g n
    __device__ __forceinline__ float whole(int64_t n, float h, float dz, float m0, float m1) const {
        float v[1] = {0.f};
        if (p.dh) load_f<TX, 1>(static_cast<const TX*>(p.dh) + m * p.lddh + n, v);
        return v[0] + r * (fmaf(dz, weight(p.v.w, p.v.w32, n, 1.f), -m0) - h * m1);
    }
};
// A block walks rows as above; what a thread would keep in registers it reads again, and the sums over the rows are added up in the
// workspace, where a walker's columns are its own.
template <class TX, class TF, bool POST>
__global__ void __launch_bounds__(1024) residual_norm_backward_wide_kernel(const BwdParams p) {
    __shared__ float red[2][32][2];
    const float inv_n = 1.f / static_cast<float>(p.N);
    float* const out = p.part ? p.part + static_cast<int64_t>(blockIdx.x) * (POST ? 4 : 3) * p.N : nullptr;
    using E = Element<TX, TF, POST>;
    for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x) {
        const E at(p, m);
        float s[2] = {0.f, 0.f}, k[2] = {0.f, 0.f}, f, h, dz;
        for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
            at(n, f, h, dz);
            const float g = dz * E::weight(p.v.w, p.v.w32, n, 1.f);
            s[0] += g;
            s[1] = fmaf(g, h, s[1]);
        }
        row_sum<1024, 2>(s, red[0]);
        const float m0 = p.center ? s[0] * inv_n : 0.f, m1 = s[1] * inv_n;
        for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
            at(n, f, h, dz);
            const float t = at.whole(n, h, dz, m0, m1), du = t * E::weight(p.v.gate, p.v.w32, n, 1.f);
            const float dx[1] = {p.scale * t}, df[1] = {du};
            if (p.dx) store_f<TX, 1>(static_cast<TX*>(p.dx) + m * p.lddx + n, dx);
            if constexpr (POST) {
                const float q = du * E::weight(p.v.pw, p.v.w32, n, 1.f);
                k[0] += q;
                k[1] = fmaf(q, f, k[1]);
            } else {
                if (p.df) store_f<TF, 1>(static_cast<TF*>(p.df) + m * p.lddf + n, df);
            }
            if (out) {
                const bool begin = m == blockIdx.x;
                const auto add = [&](int i, float v) { out[i * p.N + n] = begin ? v : out[i * p.N + n] + v; };
                add(0, dz * h);
                add(1, dz);
                add(2, t * f);
                if constexpr (POST) add(3, t);
            }
        }
        if constexpr (POST) {
            row_sum<1024, 2>(k, red[1]);
            const float c0 = p.center ? -k[0] * inv_n : 0.f, c1 = -k[1] * inv_n;
            if (p.df)
                for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
                    at(n, f, h, dz);
                    const float q = at.whole(n, h, dz, m0, m1) * E::weight(p.v.gate, p.v.w32, n, 1.f) * E::weight(p.v.pw, p.v.w32, n, 1.f);
                    const float df[1] = {at.fr * fmaf(f, c1, q + c0)};
                    store_f<TF, 1>(static_cast<TF*>(p.df) + m * p.lddf + n, df);
                }
        } else {
            __syncthreads();               // red is written again
        }
    }
}

// ---------------------------------------------------------------------------------- host
struct Width {
    int threads, elems;
};
// Threads of a row and elements of a thread; none: the wide kernel.
constexpr Width kWidths[] = {{32, 8}, {32, 16}, {128, 8}, {256, 8}, {512, 8}, {512, 16}};
int width_of(int64_t N) {
    for (int i = 0; i < 6; ++i)
        if (N <= static_cast<int64_t>(kWidths[i].threads) * kWidths[i].elems) return i;
    return 6;
}
// Walkers: all that are resident, while each still has 16 rows, since its sums go through the workspace, but one per SM at least.
struct Grid {
    int blocks, walkers;
};
Grid grid_of(int64_t M, int64_t N) {
    const int w = width_of(N), per_block = w < 6 && kWidths[w].threads == 32 ? 4 : 1, per_sm = w < 6 ? blocks_of(kWidths[w].threads) : 2;
    const int64_t all = atb::ceil_div(M, per_block), most = static_cast<int64_t>(atb::kSmCount) * per_sm;
    int64_t blocks = atb::ceil_div(M, 16 * per_block);
    if (blocks < atb::kSmCount) blocks = atb::kSmCount;
    if (blocks > most) blocks = most;
    if (blocks > all) blocks = all;
    if (blocks < 1) blocks = 1;
    return {static_cast<int>(blocks), static_cast<int>(blocks) * per_block};
}

template <class TX, class TF, int VEC, bool POST, int TPR, int ELEMS>
cudaError_t launch_rows(const BwdParams& p, cudaStream_t st) {
    constexpr int NV = ELEMS / VEC, STAGES = ahead_of<TX, TF, VEC, TPR, NV>() + 1;
    return launch_ring(residual_norm_backward_kernel<TX, TF, VEC, TPR, NV, POST>, static_cast<unsigned>(grid_of(p.M, p.N).blocks), TPR == 32 ? 128u : TPR,
                       static_cast<size_t>(STAGES) * kStage<TX, TF, VEC, TPR, NV>, st, p);
}
template <class TX, class TF, int VEC, bool POST>
cudaError_t launch(const BwdParams& p, cudaStream_t st) {
    switch (width_of(p.N)) {
        case 0: return launch_rows<TX, TF, VEC, POST, 32, 8>(p, st);
        case 1: return launch_rows<TX, TF, VEC, POST, 32, 16>(p, st);
        case 2: return launch_rows<TX, TF, VEC, POST, 128, 8>(p, st);
        case 3: return launch_rows<TX, TF, VEC, POST, 256, 8>(p, st);
        case 4: return launch_rows<TX, TF, VEC, POST, 512, 8>(p, st);
        case 5: return launch_rows<TX, TF, VEC, POST, 512, 16>(p, st);
    }
    residual_norm_backward_wide_kernel<TX, TF, POST><<<static_cast<unsigned>(grid_of(p.M, p.N).blocks), 1024, 0, st>>>(p);
    return cudaGetLastError();
}
template <class TX, class TF>
cudaError_t launch_types(const BwdParams& p, bool vec, bool post, cudaStream_t st) {
    if (vec) return post ? launch<TX, TF, 8, true>(p, st) : launch<TX, TF, 8, false>(p, st);
    return post ? launch<TX, TF, 1, true>(p, st) : launch<TX, TF, 1, false>(p, st);
}

}  // namespace

int walkers(int64_t M, int64_t N) { return grid_of(M, N).walkers; }

cudaError_t launch_backward(const BwdParams& p, Types types, bool vec, bool post, cudaStream_t stream) {
    switch (types) {
        case kBf16: return launch_types<__nv_bfloat16, __nv_bfloat16>(p, vec, post, stream);
        case kMixed: return launch_types<float, __nv_bfloat16>(p, vec, post, stream);
        default: return launch_types<float, float>(p, vec, post, stream);
    }
}

}  // namespace residual_norm
