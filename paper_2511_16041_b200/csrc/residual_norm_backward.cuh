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
// 16384 x 8192 bf16, gate, without the norm of f: 254 us (6.3 TB/s) and 9 for the sums; with it 432 (3.7 TB/s): four sums a column fill the
// registers, and instructions bind it.  8192 x 4096 bf16 77 us (5.2 TB/s) and 108 with the norm of f.
#pragma once
#include "atb_residual_norm.cuh"

namespace residual_norm {
namespace {

// Two FP32 rows of more than 4096 elements leave no room for dh beside x, f and dz twice, nor do those of an FP32 stream of more than 6144 where the
// vectors of weights need it (8192 x 8192 with a norm of f 301 us; with dh on its way and the vectors read where they are used 396): it is
// loaded where it is used.
template <class TX, class TF, int VEC, int TPR, int NV, bool POST>
constexpr bool kDirect = NV * VEC > 8 && (sizeof(TX) + sizeof(TF) == 8 || (sizeof(TX) + sizeof(TF) == 6 && POST && TPR >= 512));
template <class TX, class TF, int VEC, int TPR, int NV, bool POST>
constexpr int kStage = static_cast<int>((kDirect<TX, TF, VEC, TPR, NV, POST> ? 1 : 2) * RowSource<TX, VEC, TPR, NV>::STAGE_BYTES + 2 * RowSource<TF, VEC, TPR, NV>::STAGE_BYTES);
// Bytes of the vectors of weights in shared memory: three, where a thread's registers are full of sums (16 elements, four sums) and two stages
// of rows leave the room (read where they are used, 8192 x 6001 bf16 took 616 us instead of 264).
constexpr int kRoom = 226 * 1024;
template <class TX, class TF, int VEC, int TPR, int NV, bool POST>
__host__ __device__ constexpr int vector_bytes() {
    const int bytes = 3 * (NV * VEC / 8) * 2 * TPR * 16;
    return POST && NV * VEC == 16 && kRoom - bytes >= 2 * kStage<TX, TF, VEC, TPR, NV, POST> ? bytes : 0;
}
template <class TX, class TF, int VEC, int TPR, int NV, bool POST>
__host__ __device__ constexpr int ahead_of() {
    const int vectors = vector_bytes<TX, TF, VEC, TPR, NV, POST>();
    const int stages = (vectors ? kRoom - vectors : 208 * 1024) / (blocks_of(TPR) * kStage<TX, TF, VEC, TPR, NV, POST>);
    return stages > 4 ? 3 : stages - 1;
}

template <class TX, class TF, class TW, int VEC, int TPR, int NV, int FULL, bool POST>
__global__ void __launch_bounds__(TPR == 32 ? 128 : TPR, blocks_of(TPR)) residual_norm_backward_kernel(const BwdParams p) {
    using SX = RowSource<TX, VEC, TPR, NV>;
    using SF = RowSource<TF, VEC, TPR, NV>;
    using Shared = std::conditional_t<SX::SHARED, SX, SF>;
    constexpr bool DIRECT = kDirect<TX, TF, VEC, TPR, NV, POST>;
    constexpr int WALKERS = TPR == 32 ? 4 : 1, W = TPR / 32, AHEAD = ahead_of<TX, TF, VEC, TPR, NV, POST>(), STAGES = AHEAD + 1, CH = NV * VEC / 8;
    using At = Eight<VEC, TPR, FULL>;
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
    // The vectors that a row meets: w, gate, pw and pb.  Single elements, which are kept in FP32, are met by a and b of h = scale x + a m + b instead
    // (m = norm(f), a = gate pw, b = gate pb): one vector fewer; kept as they are in memory, the four took no more room and time than
    // the two.  They stay in registers where those have room for them beside the sums: not with 16 elements and four sums a thread, where
    // w, a and b lie in shared memory if that has the room.
    constexpr bool IN_SHARED = vector_bytes<TX, TF, VEC, TPR, NV, POST>() > 0, FOLD = POST && (VEC == 1 || IN_SHARED);
    constexpr int KEEP = IN_SHARED ? kShared : !POST || CH == 1 ? kKept : kRead;
    const uint32_t place = base + STAGES * kStage<TX, TF, VEC, TPR, NV, POST>;
    using Kept = Vector<TW, VEC, TPR, CH, FULL, KEEP>;
    const Kept w_of(N, col, p.v.w, 1.f, nullptr, 1.f, place);
    const Vector<TW, VEC, TPR, CH, FULL, KEEP, FOLD> a_of(N, col, p.v.gate, 1.f, p.v.pw, 1.f, place + Kept::BYTES);                  // gate, or a
    const Vector<TW, VEC, TPR, CH, FULL, POST && !FOLD ? KEEP : kRead> pw_of(N, col, p.v.pw, 1.f);
    const Vector<TW, VEC, TPR, CH, FULL, POST ? KEEP : kRead, FOLD> b_of(N, col, p.v.pb, 0.f, FOLD ? p.v.gate : nullptr, 1.f, place + 2 * Kept::BYTES);   // pb, or b
    const float2 zero = both(0.f), scale = both(p.scale);
    float2 s0[CH][4], s1[CH][4], s2[CH][4], s3[POST ? CH : 1][4];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            s0[c][k] = s1[c][k] = s2[c][k] = zero;
            if constexpr (POST) s3[c][k] = zero;
        }
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
        async_wait<AHEAD>();
        row_barrier<Shared, VEC, TPR>();
        // f, or norm(f), norm(h) and dz of an eight
        const auto values = [&](const At& at, float2 (&f)[4], float2 (&h)[4], float2 (&dz)[4]) {
            float2 a[4], x[4];
            at.template read<TF>(sf, stage, m, f);
            at.template read<TX>(sx, stage, m, x);
            a_of.get(at, a);
            const float2 shift = both(-mu), spread = both(r);
            if constexpr (POST) {
                float2 b[4], pw[4];
                b_of.get(at, b);
                if constexpr (!FOLD) pw_of.get(at, pw);
                const float2 f_shift = both(-fmu), f_spread = both(fr);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    f[k] = mul2(add2(f[k], f_shift), f_spread);
                    h[k] = FOLD ? fma2(f[k], a[k], b[k]) : mul2(a[k], fma2(f[k], pw[k], b[k]));
                }
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) h[k] = mul2(f[k], a[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) h[k] = mul2(add2(fma2(scale, x[k], h[k]), shift), spread);
            at.template read<TF>(sdz, stage, m, dz);
        };
        // Eight elements stay in registers over the sums, but beside four sums only single ones: else these are made again from the row in shared
        // memory, which sixteen bytes at a time costs less than the registers (8192 x 4096 with a norm of f 108 us, held 134 us).
        constexpr int HELD = CH == 1 && (VEC == 1 || !POST) ? 1 : 0;
        float2 held_f[HELD + 1][4], held_h[HELD + 1][4], held_dz[HELD + 1][4];
        float2 s_g = zero, s_gn = zero;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const At at{N, col, c};
            if (VEC == 8 && !at.in(0)) continue;
            float2 (&f)[4] = held_f[0], (&h)[4] = held_h[0], (&dz)[4] = held_dz[0], w[4];
            values(at, f, h, dz);
            w_of.get(at, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                s0[c][k] = fma2(dz[k], h[k], s0[c][k]);
                s1[c][k] = add2(s1[c][k], dz[k]);
                const float2 g = mul2(dz[k], w[k]);
                s_g = add2(s_g, g);
                s_gn = fma2(g, h[k], s_gn);
            }
        }
        float s[2] = {s_g.x + s_g.y, s_gn.x + s_gn.y};
        row_sum<TPR, 2>(s, red[0][turn]);
        // t = dh + r (dz w - m0 - n m1)
        const float2 m0 = both(p.center ? -s[0] * inv_n : 0.f), m1 = both(-s[1] * inv_n), spread = both(r);
        float2 q[POST ? CH : 1][4], k_q = zero, k_qm = zero;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const At at{N, col, c};
            if (VEC == 8 && !at.in(0)) continue;
            float2 (&f)[4] = held_f[0], (&h)[4] = held_h[0], (&d)[4] = held_dz[0], w[4];
            if constexpr (!HELD) values(at, f, h, d);
            w_of.get(at, w);
#pragma unroll
            for (int k = 0; k < 4; ++k) d[k] = mul2(spread, fma2(h[k], m1, fma2(d[k], w[k], m0)));
            if (has_dh) {
                if constexpr (DIRECT) at.template load<TX>(static_cast<const TX*>(p.dh) + m * p.lddh, w);
                else at.template read<TX>(sdh, stage, m, w);
#pragma unroll
                for (int k = 0; k < 4; ++k) d[k] = add2(d[k], w[k]);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                s2[c][k] = fma2(d[k], f[k], s2[c][k]);
                if constexpr (POST) s3[c][k] = add2(s3[c][k], d[k]);
                w[k] = mul2(scale, d[k]);
            }
            if (p.dx) at.template store<TX>(static_cast<TX*>(p.dx) + m * p.lddx, w);
            a_of.get(at, w);
            if constexpr (POST) {
                float2 pw[4];
                if constexpr (!FOLD) pw_of.get(at, pw);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    q[c][k] = FOLD ? mul2(d[k], w[k]) : mul2(mul2(d[k], w[k]), pw[k]);
                    k_q = add2(k_q, q[c][k]);
                    k_qm = fma2(q[c][k], f[k], k_qm);
                }
            } else if (p.df) {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = mul2(w[k], d[k]);
                at.template store<TF>(static_cast<TF*>(p.df) + m * p.lddf, w);
            }
        }
        if constexpr (POST) {
            float k[2] = {k_q.x + k_q.y, k_qm.x + k_qm.y};
            row_sum<TPR, 2>(k, red[1][turn]);
            const float2 c0 = both(p.center ? -k[0] * inv_n : 0.f), c1 = both(-k[1] * inv_n), shift = both(-fmu), fspread = both(fr);
            if (p.df)
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const At at{N, col, c};
                    if (VEC == 8 && !at.in(0)) continue;
                    float2 (&f)[4] = held_f[0];
                    if constexpr (!HELD) {
                        at.template read<TF>(sf, stage, m, f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) f[e] = mul2(add2(f[e], shift), fspread);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] = mul2(fspread, fma2(f[e], c1, add2(q[c][e], c0)));
                    at.template store<TF>(static_cast<TF*>(p.df) + m * p.lddf, f);
                }
        }
        // the row's stage is the next to be filled, by other threads than those that have just read it
        row_barrier<Shared, VEC, TPR>();
        mu = next[0]; r = next[1]; fmu = next[2]; fr = next[3];
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    if (p.part) {                          // a walker's sums: [walker][sums][N]
        float* const out = p.part + first * (POST ? 4 : 3) * p.N;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const At at{N, col, c};
            at.template store<float>(out, s0[c]);
            at.template store<float>(out + p.N, s1[c]);
            at.template store<float>(out + 2 * p.N, s2[c]);
            if constexpr (POST) at.template store<float>(out + 3 * p.N, s3[c]);
        }
    }
}

// ---------------------------------------------------------------------------------- any width
// One element's f (or norm(f)) and norm(h).
template <class TX, class TF, class TW, bool POST>
struct Element {
    const BwdParams& p;
    int64_t m;
    float mu, r, fmu, fr;
    __device__ __forceinline__ Element(const BwdParams& p_, int64_t m_) : p(p_), m(m_), mu(p_.stats[m_]), r(p_.stats[p_.M + m_]), fmu(0.f), fr(1.f) {
        if constexpr (POST) { fmu = p.stats[2 * p.M + m]; fr = p.stats[3 * p.M + m]; }
    }
    static __device__ __forceinline__ float weight(const void* w, int64_t n, float none) {
        float v[1];
        weights<TW, 1>(w, static_cast<int>(n), none, v);
        return v[0];
    }
    __device__ __forceinline__ void operator()(int64_t n, float& f, float& h, float& dz) const {
        float v[1];
        load_f<TF, 1>(static_cast<const TF*>(p.f) + m * p.ldf + n, v);
        f = v[0];
        h = f;
        if constexpr (POST) {
            f = (f - fmu) * fr;
            h = fmaf(f, weight(p.v.pw, n, 1.f), weight(p.v.pb, n, 0.f));
        }
        load_f<TX, 1>(static_cast<const TX*>(p.x) + m * p.ldx + n, v);
        h = (fmaf(p.scale, v[0], weight(p.v.gate, n, 1.f) * h) - mu) * r;
        load_f<TF, 1>(static_cast<const TF*>(p.dz) + m * p.lddz + n, v);
        dz = v[0];
    }
    // t from the means of g and g n
    __device__ __forceinline__ float whole(int64_t n, float h, float dz, float m0, float m1) const {
        float v[1] = {0.f};
        if (p.dh) load_f<TX, 1>(static_cast<const TX*>(p.dh) + m * p.lddh + n, v);
        return v[0] + r * (fmaf(dz, weight(p.v.w, n, 1.f), -m0) - h * m1);
    }
};
// A block walks rows as above; what a thread would keep in registers it reads again, and the sums over the rows are added up in the
// workspace, where a walker's columns are its own.
template <class TX, class TF, class TW, bool POST>
__global__ void __launch_bounds__(1024) residual_norm_backward_wide_kernel(const BwdParams p) {
    __shared__ float red[2][32][2];
    const float inv_n = 1.f / static_cast<float>(p.N);
    float* const out = p.part ? p.part + static_cast<int64_t>(blockIdx.x) * (POST ? 4 : 3) * p.N : nullptr;
    using E = Element<TX, TF, TW, POST>;
    for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x) {
        const E at(p, m);
        float s[2] = {0.f, 0.f}, k[2] = {0.f, 0.f}, f, h, dz;
        for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
            at(n, f, h, dz);
            const float g = dz * E::weight(p.v.w, n, 1.f);
            s[0] += g;
            s[1] = fmaf(g, h, s[1]);
        }
        row_sum<1024, 2>(s, red[0]);
        const float m0 = p.center ? s[0] * inv_n : 0.f, m1 = s[1] * inv_n;
        for (int64_t n = threadIdx.x; n < p.N; n += 1024) {
            at(n, f, h, dz);
            const float t = at.whole(n, h, dz, m0, m1), du = t * E::weight(p.v.gate, n, 1.f);
            const float dx[1] = {p.scale * t}, df[1] = {du};
            if (p.dx) store_f<TX, 1>(static_cast<TX*>(p.dx) + m * p.lddx + n, dx);
            if constexpr (POST) {
                const float q = du * E::weight(p.v.pw, n, 1.f);
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
                    const float q = at.whole(n, h, dz, m0, m1) * E::weight(p.v.gate, n, 1.f) * E::weight(p.v.pw, n, 1.f);
                    const float df[1] = {at.fr * fmaf(f, c1, q + c0)};
                    store_f<TF, 1>(static_cast<TF*>(p.df) + m * p.lddf + n, df);
                }
        } else {
            __syncthreads();               // red is written again
        }
    }
}

// ---------------------------------------------------------------------------------- host
template <class TX, class TF, class TW, int VEC, bool POST, int W>
cudaError_t launch_rows(const BwdParams& p, cudaStream_t st) {
    constexpr int TPR = kWidths[W].threads, NV = kWidths[W].elems / VEC, STAGES = ahead_of<TX, TF, VEC, TPR, NV, POST>() + 1;
    constexpr int FULL = full_of(TPR, kWidths[W].elems, VEC, W > 0 ? kWidths[W > 0 ? W - 1 : 0].threads * kWidths[W > 0 ? W - 1 : 0].elems : 0);
    return launch_ring<&residual_norm_backward_kernel<TX, TF, TW, VEC, TPR, NV, FULL, POST>>(static_cast<unsigned>(p.blocks), TPR == 32 ? 128u : TPR,
                                                                                             static_cast<size_t>(STAGES) * kStage<TX, TF, VEC, TPR, NV, POST> + vector_bytes<TX, TF, VEC, TPR, NV, POST>(), st, p);
}
template <class TX, class TF, class TW, int VEC, bool POST>
cudaError_t launch(const BwdParams& p, cudaStream_t st) {
    switch (width_of(p.N)) {
        case 0: return launch_rows<TX, TF, TW, VEC, POST, 0>(p, st);
        case 1: return launch_rows<TX, TF, TW, VEC, POST, 1>(p, st);
        case 2: return launch_rows<TX, TF, TW, VEC, POST, 2>(p, st);
        case 3: return launch_rows<TX, TF, TW, VEC, POST, 3>(p, st);
        case 4: return launch_rows<TX, TF, TW, VEC, POST, 4>(p, st);
        case 5: return launch_rows<TX, TF, TW, VEC, POST, 5>(p, st);
        case 6: return launch_rows<TX, TF, TW, VEC, POST, 6>(p, st);
        case 7: return launch_rows<TX, TF, TW, VEC, POST, 7>(p, st);
        case 8: return launch_rows<TX, TF, TW, VEC, POST, 8>(p, st);
        case 9: return launch_rows<TX, TF, TW, VEC, POST, 9>(p, st);
    }
    residual_norm_backward_wide_kernel<TX, TF, TW, POST><<<static_cast<unsigned>(p.blocks), 1024, 0, st>>>(p);
    return cudaGetLastError();
}
template <class TX, class TF, class TW>
cudaError_t launch_types(const BwdParams& p, bool vec, bool post, cudaStream_t st) {
    if (vec) return post ? launch<TX, TF, TW, 8, true>(p, st) : launch<TX, TF, TW, 8, false>(p, st);
    return post ? launch<TX, TF, TW, 1, true>(p, st) : launch<TX, TF, TW, 1, false>(p, st);
}
template <class TW>
cudaError_t launch_backward(const BwdParams& p, Types types, bool vec, bool post, cudaStream_t st) {
    switch (types) {
        case kBf16: return launch_types<__nv_bfloat16, __nv_bfloat16, TW>(p, vec, post, st);
        case kMixed: return launch_types<float, __nv_bfloat16, TW>(p, vec, post, st);
        default: return launch_types<float, float, TW>(p, vec, post, st);
    }
}

}  // namespace
}  // namespace residual_norm
