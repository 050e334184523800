// The gated delta rule, forward: what a chunk's tokens do to each other (merit_delta_prepare), chunk after chunk
// (merit_delta_chunks), one token (merit_delta_token).  The formulas stand in delta.h.
#pragma once

#include "delta.h"

namespace merit {
namespace delta {

// ---------------------------------------------------------------------------
// chunks side by side: a workgroup a chunk of a head
// ---------------------------------------------------------------------------
// Forward it leaves X = (1 + N diag(b))^-1 and P = scale f o Q K^T, rows side by side; backward the transposes of
// (1 + diag(b) N)^-1 and P.  Blocks of 16 x 16 above the diagonal are not written but where a product of 32 reads them.
template <typename T, int KF, bool BACK>
__global__ __launch_bounds__(NT) void merit_delta_prepare(DeltaParams p)
{
    constexpr int NK = Terms<T>::n, NP = mix_terms<T>(BACK);
    __shared__ __attribute__((aligned(16))) __bf16 kmem[Tile<NK, C, KF * 32>::bytes / 2];
    __shared__ __attribute__((aligned(16))) float a[C][C + 4];
    __shared__ double G[C];
    __shared__ float beta[C], invk[C], invq[C];
    __shared__ int bad;             // the first token whose row of the triangular matrix is not finite
    const Tile<NK, C, KF * 32> kt{kmem};

    const uint32_t id = blockIdx.x, h = id % (uint32_t)p.H, bi = id / (uint32_t)p.H;
    const uint32_t i = bi % (uint32_t)p.n;
    const int64_t b = bi / (uint32_t)p.n, t0 = (int64_t)i * C;
    const int kh = (int)h / p.each, m = min(C, tokens_of(p, b) - (int)t0);
    if (m <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quad = lane >> 4;
    float *scal = p.scal + (int64_t)id * SCALAR_FLOATS;

    // Two rows' loads in a wavefront: keys to LDS, their squares' sums over the lanes of a row
    ChunkRows<T, KF> kr;
    kr.load(p.k, b, t0, m, kh, p.Dk, p.wide_qk);
    const T *qrow = static_cast<const T *>(p.q.data) + b * p.q.s0 + (t0 + 16 * wave + l16) * p.q.s1 + (int64_t)kh * p.Dk;
    Eight<T> qe[KF];
#pragma unroll
    for (int f = 0; f < KF; ++f) {
        qe[f] = zero8<T>();
        if (16 * wave + l16 < m) qe[f] = load8<T>(qrow, 32 * f + 8 * quad, p.Dk, p.wide_qk);
    }
    if (wave == 0) {
        double g = 0.0;
        float bt = 0.0f;
        if (lane < m) {
            if (p.g.data) g = (double)static_cast<const float *>(p.g.data)[b * p.g.s0 + (t0 + lane) * p.g.s1 + h];
            if (g < -1000.0) g = -1000.0;       // (no decay of fp32 is that small: -inf, which has no differences, included)
            const int64_t at = b * p.beta.s0 + (t0 + lane) * p.beta.s1 + h;
            bt = p.beta_f32 ? static_cast<const float *>(p.beta.data)[at] : (float)static_cast<const T *>(p.beta.data)[at];
        }
#pragma unroll
        for (int s = 1; s < C; s *= 2) {
            const double o = __shfl_up(g, s);
            if (lane >= s) g += o;
        }
        G[lane] = g;
        beta[lane] = bt;
    }
    if (p.unit) {
#pragma unroll
        for (int u = 0; u < ChunkRows<T, KF>::units; ++u) {
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf((float)kr.e[u].v[e], (float)kr.e[u].v[e], s);
            s = sum_lanes(s, KF * 4);
            if (tid % (KF * 4) == 0) invk[(tid + u * NT) / (KF * 4)] = 1.0f / sqrtf(s + MERIT_DELTA_EPS);
        }
        float s = 0.0f;
#pragma unroll
        for (int f = 0; f < KF; ++f)
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf((float)qe[f].v[e], (float)qe[f].v[e], s);
        s += lane_xor<4>(s);
        s += lane_xor<5>(s);
        if (quad == 0) invq[16 * wave + l16] = 1.0f / sqrtf(s + MERIT_DELTA_EPS);
    } else if (tid < C) {
        invk[tid] = invq[tid] = 1.0f;
    }
    if (tid == 0) bad = C;
    kr.store(kt);
    __syncthreads();

    if (tid < C) {
        const double g = G[tid], last = G[C - 1];
        const float in = exp_of(g);
        scal[IN_K * C + tid] = in * invk[tid];
        scal[BETA * C + tid] = beta[tid];
        scal[OUT_K * C + tid] = exp_of(last - g) * invk[tid];
        scal[IN_Q * C + tid] = p.scale * in * invq[tid];
        scal[INV_K * C + tid] = invk[tid];
        scal[INV_Q * C + tid] = invq[tid];
        reinterpret_cast<double *>(scal + SCALARS * C)[tid] = g;
    }

    // Rows or columns 16 wave .. of K K^T and Q K^T, up to the diagonal's block
    __bf16 *mix = static_cast<__bf16 *>(p.mix) + (int64_t)id * NP * C * C;
    bf16x8 qa[KF][NK], ka[KF][NK];
#pragma unroll
    for (int f = 0; f < KF; ++f) {
        terms8<T>(qe[f], qa[f]);
        kt.rows(16 * wave, 32 * f, ka[f]);
    }
    for (int jb = 0; jb < 4; ++jb) {
        f32x4 kk = {0, 0, 0, 0}, qk = {0, 0, 0, 0};
        if (jb <= wave)
#pragma unroll
            for (int f = 0; f < KF; ++f) {
                bf16x8 o[NK];
                kt.rows(16 * jb, 32 * f, o);
                // backward: the lane has a column of four rows, whose transpose lies side by side; forward the other way round
                if constexpr (BACK) {
                    multiply<3>(kk, ka[f], o);
                    multiply<3>(qk, qa[f], o);
                } else {
                    multiply<3>(kk, o, ka[f]);
                    multiply<3>(qk, o, qa[f]);
                }
            }
        bf16x4 out[NP];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = BACK ? 16 * wave + 4 * quad + r : 16 * wave + l16;          // the token that reads
            const int j = BACK ? 16 * jb + l16 : 16 * jb + 4 * quad + r;              // the token that was written
            const float f = j <= t ? exp_of(G[t] - G[j]) : 0.0f;
            float w = j < t ? f * invk[t] * invk[j] * (BACK ? beta[t] : beta[j]) * kk[r] : 0.0f;
            if (!isfinite(w)) {     // (0 times it would reach the tokens before)
                atomicMin(&bad, t);
                w = 0.0f;
            }
            // (backward the columns of the inverse are wanted side by side, forward its rows)
            if constexpr (BACK) a[t][j] = w;
            else a[j][t] = w;
            __bf16 s[NP];
            split<NP>(j <= t ? f * p.scale * invq[t] * invk[j] * qk[r] : 0.0f, s);
#pragma unroll
            for (int n = 0; n < NP; ++n) out[n][r] = s[n];
        }
        if (jb <= (wave | 1))
#pragma unroll
            for (int n = 0; n < NP; ++n) {
                __bf16 *to = mix + n * C * C +
                             (BACK ? (16 * jb + l16) * C + 16 * wave + 4 * quad : (16 * wave + l16) * C + 16 * jb + 4 * quad);
                *reinterpret_cast<bf16x4 *>(to) = out[n];
            }
    }
    __syncthreads();

    // The inverse: lane c has column c (backward), or row c (forward), and takes one value after the other
    if (wave == 0) {
        float x[C];
#pragma unroll
        for (int s = 0; s < C; ++s) {
            const int r = BACK ? s : C - 1 - s;
            float v0 = r == lane ? 1.0f : 0.0f, v1 = 0.0f, v2 = 0.0f, v3 = 0.0f;
            if constexpr (BACK) {
#pragma unroll
                for (int j = 0; j < r; j += 4) {
                    const f32x4 w = *reinterpret_cast<const f32x4 *>(&a[r][j]);
                    v0 = fmaf(-w[0], x[j], v0);
                    if (j + 1 < r) v1 = fmaf(-w[1], x[j + 1], v1);
                    if (j + 2 < r) v2 = fmaf(-w[2], x[j + 2], v2);
                    if (j + 3 < r) v3 = fmaf(-w[3], x[j + 3], v3);
                }
            } else {
#pragma unroll
                for (int j = r / 4 * 4; j < C; j += 4) {
                    const f32x4 w = *reinterpret_cast<const f32x4 *>(&a[r][j]);
                    if (j > r) v0 = fmaf(-w[0], x[j], v0);
                    if (j + 1 > r) v1 = fmaf(-w[1], x[j + 1], v1);
                    if (j + 2 > r) v2 = fmaf(-w[2], x[j + 2], v2);
                    if (j + 3 > r) v3 = fmaf(-w[3], x[j + 3], v3);
                }
            }
            x[r] = (v0 + v1) + (v2 + v3);
        }
        __bf16 *to = static_cast<__bf16 *>(p.tri) + (int64_t)id * 3 * C * C + lane * C;
        const bool lost = !BACK && lane >= bad;
#pragma unroll
        for (int c = 0; c < C; c += 8) {
            float e[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) e[k] = lost ? __builtin_nanf("") : x[c + k];
            bf16x8 o[3];
            split8<3>(e, o);
#pragma unroll
            for (int n = 0; n < 3; ++n) *reinterpret_cast<bf16x8 *>(to + n * C * C + c) = o[n];
        }
    }
}

// ---------------------------------------------------------------------------
// one chunk after the other: a workgroup 16 NC columns of a head's state
// ---------------------------------------------------------------------------
// The columns of a state do not depend on each other.  A wavefront has 16 of the chunk's tokens, and 16 or 32 rows of the state
// in registers, from which it goes to LDS in three terms for the next chunk's products.
template <typename T, int KF, int NC>
__global__ __launch_bounds__(NT) void merit_delta_chunks(DeltaParams p)
{
    constexpr int NK = Terms<T>::n, NP = mix_terms<T>(false), RT = KF < 2 ? 1 : KF / 2, ORD = NP;
    extern __shared__ __attribute__((aligned(16))) __bf16 smem[];
    typedef Tile<NK, C, KF * 32> TK;
    typedef Tile<3, NC * 16, KF * 32> TS;
    typedef Tile<3, NC * 16, C> TX;
    typedef Tile<NP, NC * 16, C> TU;
    const TK kt{smem};
    const TS st{kt.at + TK::bytes / 2};
    const TX xt{st.at + TS::bytes / 2}, ot{xt.at + TX::bytes / 2};
    const TU ut{ot.at + TX::bytes / 2};
    // The first token of a chunk from which a column is not finite: such values go into products as zeros, because those of
    // earlier tokens have them too, times 0.  (Set once: the chunks behind it start from a state that is not finite.)
    __shared__ int bad[NC * 16];

    const uint32_t id = blockIdx.x, h = id / (uint32_t)p.slices % (uint32_t)p.H;
    const int64_t b = id / (uint32_t)p.slices / (uint32_t)p.H;
    const int c0 = (int)(id % (uint32_t)p.slices) * NC * 16, kh = (int)h / p.each;
    const int len = tokens_of(p, b), n = (len + C - 1) / C;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quad = lane >> 4;
    const int row4 = 16 * wave + 4 * quad;                     // the first of a lane's four tokens in a result of 16 x 16
    const int64_t head = b * p.H + h, Dv = p.Dv;
    const bool has_rows = wave < 2 * KF;

    f32x4 S[RT][NC];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int dk = 16 * (wave + 4 * rt) + 4 * quad + r, dv = c0 + 16 * ct + l16;
                S[rt][ct][r] = p.h0 && dk < p.Dk && dv < Dv ? p.h0[(head * p.Dk + dk) * Dv + dv] : 0.0f;
            }
    auto state_to_lds = [&]() __attribute__((always_inline)) {
        if (has_rows)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int ct = 0; ct < NC; ++ct) {
                    const float e[4] = {S[rt][ct][0], S[rt][ct][1], S[rt][ct][2], S[rt][ct][3]};
                    st.put4(16 * ct + l16, 16 * (wave + 4 * rt) + 4 * quad, e);
                }
    };
    auto state_to = [&](float *out) __attribute__((always_inline)) {
        if (has_rows)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int dk = 16 * (wave + 4 * rt) + 4 * quad + r, dv = c0 + 16 * ct + l16;
                        if (dk < p.Dk && dv < Dv) out[dk * Dv + dv] = S[rt][ct][r];
                    }
    };

    ChunkRows<T, KF> kr;
    if (n > 0) kr.load(p.k, b, 0, min(C, len), kh, p.Dk, p.wide_qk);
    if (tid < NC * 16) bad[tid] = C;
    state_to_lds();
    for (int i = 0; i < n; ++i) {
        const int64_t t0 = (int64_t)i * C, chunk = (b * p.n + i) * p.H + h;
        const int m = min(C, len - (int)t0);
        const float *scal = p.scal + chunk * SCALAR_FLOATS;
        kr.store(kt);
        __syncthreads();
        if (i + 1 < n) kr.load(p.k, b, t0 + C, min(C, len - (int)t0 - C), kh, p.Dk, p.wide_qk);

        // K S and Q S
        const T *qrow = static_cast<const T *>(p.q.data) + b * p.q.s0 + (t0 + 16 * wave + l16) * p.q.s1 + (int64_t)kh * p.Dk;
        Eight<T> qe[KF];
#pragma unroll
        for (int f = 0; f < KF; ++f) {
            qe[f] = zero8<T>();
            if (16 * wave + l16 < m) qe[f] = load8<T>(qrow, 32 * f + 8 * quad, p.Dk, p.wide_qk);
        }
        float v[NC][4];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int dv = c0 + 16 * ct + l16;
                v[ct][r] = row4 + r < m && dv < Dv
                               ? (float)static_cast<const T *>(p.v.data)[b * p.v.s0 + (t0 + row4 + r) * p.v.s1 + h * Dv + dv] : 0.0f;
            }
        const f32x4 in_k = *reinterpret_cast<const f32x4 *>(scal + IN_K * C + row4);
        const f32x4 in_q = *reinterpret_cast<const f32x4 *>(scal + IN_Q * C + row4);
        const f32x4 out_k = *reinterpret_cast<const f32x4 *>(scal + OUT_K * C + row4);
        const f32x4 beta = *reinterpret_cast<const f32x4 *>(scal + BETA * C + row4);
        const float whole = exp_of(reinterpret_cast<const double *>(scal + SCALARS * C)[C - 1]);
        bf16x8 tri[2][3], mix[2][NP];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            const int64_t at = (16 * wave + l16) * C + 32 * f + 8 * quad;
            if (2 * f > wave) continue;
#pragma unroll
            for (int k = 0; k < 3; ++k)
                tri[f][k] = *reinterpret_cast<const bf16x8 *>(static_cast<const __bf16 *>(p.tri) + (chunk * 3 + k) * C * C + at);
#pragma unroll
            for (int k = 0; k < NP; ++k)
                mix[f][k] = *reinterpret_cast<const bf16x8 *>(static_cast<const __bf16 *>(p.mix) + (chunk * NP + k) * C * C + at);
        }

        f32x4 R[NC], Y[NC];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) R[ct] = Y[ct] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int f = 0; f < KF; ++f) {
            bf16x8 ka[NK], qa[NK];
            kt.rows(16 * wave, 32 * f, ka);
            terms8<T>(qe[f], qa);
#pragma unroll
            for (int ct = 0; ct < NC; ++ct) {
                bf16x8 s[3];
                st.rows(16 * ct, 32 * f, s);
                multiply<3>(R[ct], ka, s);
                multiply<ORD>(Y[ct], qa, s);
            }
        }
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            float e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                e[r] = fmaf(-in_k[r], R[ct][r], v[ct][r]);
                if (!isfinite(e[r])) {
                    atomicMin(&bad[16 * ct + l16], row4 + r);
                    e[r] = 0.0f;
                }
            }
            xt.put4(16 * ct + l16, row4, e);
        }
        __syncthreads();

        // d, u
        f32x4 D[NC];
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            D[ct] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                if (2 * f > wave) continue;
                bf16x8 x[3];
                xt.rows(16 * ct, 32 * f, x);
                multiply<3>(D[ct], tri[f], x);
            }
            float u[4], o[4];
            const int from = bad[16 * ct + l16];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (row4 + r >= from) D[ct][r] = __builtin_nanf("");
                u[r] = beta[r] * D[ct][r];
                if (!isfinite(u[r])) {
                    atomicMin(&bad[16 * ct + l16], row4 + r);
                    u[r] = 0.0f;
                }
                o[r] = out_k[r] * u[r];
            }
            ut.put4(16 * ct + l16, row4, u);
            ot.put4(16 * ct + l16, row4, o);
        }
        if (p.states) {
            float *out = p.states + chunk * (p.Dk + C) * Dv;
            state_to(out);
#pragma unroll
            for (int ct = 0; ct < NC; ++ct)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int dv = c0 + 16 * ct + l16;
                    if (dv < Dv) out[(p.Dk + row4 + r) * Dv + dv] = D[ct][r];
                }
        }
        __syncthreads();

        // y, and the state behind the chunk
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            f32x4 y = {0, 0, 0, 0};
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                if (2 * f > wave) continue;
                bf16x8 u[NP];
                ut.rows(16 * ct, 32 * f, u);
                multiply<ORD>(y, mix[f], u);
            }
            const int dv = c0 + 16 * ct + l16, from = bad[16 * ct + l16];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float f = row4 + r >= from ? __builtin_nanf("") : fmaf(in_q[r], Y[ct][r], y[r]);
                if (dv < Dv && t0 + row4 + r < p.L)
                    static_cast<T *>(p.y.data)[b * p.y.s0 + (t0 + row4 + r) * p.y.s1 + h * Dv + dv] = (T)(row4 + r < m ? f : 0.0f);
            }
        }
        if (has_rows)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                bf16x8 ka[2][NK];
#pragma unroll
                for (int f = 0; f < 2; ++f) kt.cols(32 * f, 16 * (wave + 4 * rt), ka[f]);
#pragma unroll
                for (int ct = 0; ct < NC; ++ct) {
                    f32x4 s = S[rt][ct] * whole;
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        bf16x8 o[3];
                        ot.rows(16 * ct, 32 * f, o);
                        multiply<3>(s, ka[f], o);
                    }
                    if (bad[16 * ct + l16] < C) s = f32x4{1, 1, 1, 1} * __builtin_nanf("");
                    S[rt][ct] = s;
                }
            }
        state_to_lds();
        __syncthreads();
    }
    if (p.h_last) state_to(p.h_last + head * p.Dk * Dv);
    // zeros behind the sequence's last chunk
    const int cols = min(NC * 16, (int)Dv - c0);
    for (int64_t u = tid; u < (p.L - (int64_t)n * C) * cols; u += NT) {
        const int64_t t = (int64_t)n * C + u / cols;
        static_cast<T *>(p.y.data)[b * p.y.s0 + t * p.y.s1 + h * Dv + c0 + u % cols] = (T)0.0f;
    }
}

// ---------------------------------------------------------------------------
// one token
// ---------------------------------------------------------------------------
// Bound by memory: the state is read once and held in registers.  y = q.S_t = a q.S_{t-1} + (q.k) u, so both sums over the
// state's rows come from the one pass.  A workgroup has `lanes` vectors of V columns, NT / lanes threads share a column's rows.
template <typename T, int V, int ROWS>
__global__ __launch_bounds__(NT) void merit_delta_token(DeltaParams p, int lanes, int tiles)
{
    __shared__ float qk[2][MERIT_DELTA_MAX_KEYS], sums[3][4], part[2][NT][V];
    const int tid = threadIdx.x, groups = NT / lanes, group = tid / lanes, lane = tid % lanes;
    const uint32_t id = blockIdx.x;
    const int64_t head = id / (uint32_t)tiles, b = head / p.H;
    const int h = (int)(head % p.H), kh = h / p.each, c = ((int)(id % (uint32_t)tiles) * lanes + lane) * V;
    const bool in = c < p.Dv;
    const int64_t base = head * p.Dk * p.Dv + c;

    vec_t<float, V> S[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = group + j * groups;
        S[j] = in && r < p.Dk ? load_vec<float, V>(p.h0, base + (int64_t)r * p.Dv) : vec_t<float, V>{};
    }
    // q and k of the head: one value a thread, and the three sums over them
    const int d = tid & (MERIT_DELTA_MAX_KEYS - 1);
    static_assert(NT == 2 * MERIT_DELTA_MAX_KEYS, "");
    float x = 0.0f;
    if (d < p.Dk) {
        const Rows &w = tid < MERIT_DELTA_MAX_KEYS ? p.q : p.k;
        x = (float)static_cast<const T *>(w.data)[b * w.s0 + (int64_t)kh * p.Dk + d];
    }
    qk[tid / MERIT_DELTA_MAX_KEYS][d] = x;
    const float own = sum_lanes(x * x, 64);
    if ((tid & 63) == 0) sums[0][tid >> 6] = own;
    __syncthreads();
    if (tid < MERIT_DELTA_MAX_KEYS) {
        const float both = sum_lanes(qk[0][d] * qk[1][d], 64);
        if ((tid & 63) == 0) sums[1][tid >> 6] = both;
    }
    __syncthreads();
    const float iq = p.unit ? 1.0f / sqrtf(sums[0][0] + sums[0][1] + MERIT_DELTA_EPS) : 1.0f;
    const float ik = p.unit ? 1.0f / sqrtf(sums[0][2] + sums[0][3] + MERIT_DELTA_EPS) : 1.0f;
    const float dot = (sums[1][0] + sums[1][1]) * iq * ik;

    float sk[V], sq[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sk[e] = sq[e] = 0.0f;
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = group + j * groups;
        if (r >= p.Dk) continue;
        const float kv = qk[1][r], qv = qk[0][r];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            sk[e] = fmaf(kv, at<float, V>(S[j], e), sk[e]);
            sq[e] = fmaf(qv, at<float, V>(S[j], e), sq[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
        part[0][tid][e] = sk[e];
        part[1][tid][e] = sq[e];
    }
    __syncthreads();
    if (!in) return;
    const float decay = p.g.data ? exp_of((double)static_cast<const float *>(p.g.data)[b * p.g.s0 + h]) : 1.0f;
    const int64_t at_beta = b * p.beta.s0 + h;
    const float beta = p.beta_f32 ? static_cast<const float *>(p.beta.data)[at_beta] : (float)static_cast<const T *>(p.beta.data)[at_beta];
    float u[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float k = 0.0f, q = 0.0f;
        for (int g = 0; g < groups; ++g) {
            k += part[0][g * lanes + lane][e];
            q += part[1][g * lanes + lane][e];
        }
        const float v = (float)static_cast<const T *>(p.v.data)[b * p.v.s0 + (int64_t)h * p.Dv + c + e];
        u[e] = beta * fmaf(-decay * ik, k, v);
        if (group == 0)
            static_cast<T *>(p.y.data)[b * p.y.s0 + (int64_t)h * p.Dv + c + e] = (T)(p.scale * fmaf(dot, u[e], decay * iq * q));
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = group + j * groups;
        if (r >= p.Dk) continue;
        const float kv = qk[1][r] * ik;
        vec_t<float, V> o;
#pragma unroll
        for (int e = 0; e < V; ++e) put<float, V>(o, e, fmaf(kv, u[e], decay * at<float, V>(S[j], e)));
        store_vec<float, V>(p.h_last, base + (int64_t)r * p.Dv, o);
    }
}

template <typename T, int KF, int NC> hipError_t forward_chunks(DeltaParams p, hipStream_t s)
{
    constexpr int NK = Terms<T>::n, NP = mix_terms<T>(false);
    constexpr int lds = Tile<NK, C, KF * 32>::bytes + Tile<3, NC * 16, KF * 32>::bytes + 2 * Tile<3, NC * 16, C>::bytes +
                        Tile<NP, NC * 16, C>::bytes;
    static_assert(lds <= 160 * 1024, "");
    p.slices = (int)((p.Dv + 16 * NC - 1) / (16 * NC));
    merit_delta_chunks<T, KF, NC><<<(unsigned)(p.B * p.H * p.slices), NT, lds, s>>>(p);
    return hipGetLastError();
}
template <typename T, int KF> hipError_t forward_of(const DeltaParams &p, hipStream_t s)
{
    if (p.n > 0) {
        merit_delta_prepare<T, KF, false><<<(unsigned)(p.B * p.n * p.H), NT, 0, s>>>(p);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return p.Dv <= 16 ? forward_chunks<T, KF, 1>(p, s) : forward_chunks<T, KF, 2>(p, s);
}
template <typename T> hipError_t forward_typed(const DeltaParams &p, hipStream_t s)
{
    return p.Dk <= 32 ? forward_of<T, 1>(p, s) : p.Dk <= 64 ? forward_of<T, 2>(p, s) : forward_of<T, 4>(p, s);
}

template <typename T> hipError_t prepare_back_typed(const DeltaParams &p, hipStream_t s)
{
    const unsigned grid = (unsigned)(p.B * p.n * p.H);
    if (p.Dk <= 32) merit_delta_prepare<T, 1, true><<<grid, NT, 0, s>>>(p);
    else if (p.Dk <= 64) merit_delta_prepare<T, 2, true><<<grid, NT, 0, s>>>(p);
    else merit_delta_prepare<T, 4, true><<<grid, NT, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T> hipError_t token_typed(const DeltaParams &p, hipStream_t s)
{
    const int v = p.wide_state ? 4 : 1;
    int lanes = 16;
    while (lanes < 32 && lanes * v < p.Dv) lanes *= 2;
    const int tiles = (p.Dv + lanes * v - 1) / (lanes * v);
    const unsigned grid = (unsigned)(p.B * p.H * tiles);
    if (v == 4) merit_delta_token<T, 4, 16><<<grid, NT, 0, s>>>(p, lanes, tiles);
    else merit_delta_token<T, 1, 16><<<grid, NT, 0, s>>>(p, lanes, tiles);
    return hipGetLastError();
}

}  // namespace delta
}  // namespace merit
