// The gated delta rule, backward (the formulas and the representation of operands: delta.h).  With Z the gradient of the state
// behind a chunk, T = (1 + diag(b) N)^-1, K and Q of unit length (Q scaled), i = exp(G), o = exp(G_C - G):
//     x = T^T (P^T dy + o K Z),   dv = b x,   Z_before = exp(G_C) Z + Q^T (i dy) - K^T (i dv)              one chunk after the other
//     dQ = i (dy S_0^T) + (f o dy u^T) K                                                                   chunks side by side
//     dK = rows + cols,  rows = M K - i (dv S_0^T),  cols = (f o dy u^T)^T Q + M^T K + o (u Z^T),  M = -b f o (x u^T) below the diagonal
//     db = x.d,   dG = Q.dQ + K.rows - K.cols, at the last token besides exp(G_C) <S_0, Z> + K.(o u Z^T),   dg_t = sum of dG from t on
// d and S_0 come from the forward pass.
#pragma once

#include "delta_forward.h"

namespace merit {
namespace delta {

// ---------------------------------------------------------------------------
// one chunk after the other, from the last: a wavefront 16 columns of a head's Z
// ---------------------------------------------------------------------------
// Split as merit_delta_chunks is: a wavefront has its columns of Z and of all tokens in registers, LDS holds K, Q and the transposes
// of the triangular matrices, of which a row of blocks begins at the diagonal.
template <typename T, int KF, bool WIDE>
__global__ __launch_bounds__(NT) void merit_delta_back_chunks(DeltaParams p)
{
    constexpr int NK = Terms<T>::n, NP = mix_terms<T>(true), RT = C / 16, DT = 2 * KF;
    extern __shared__ __attribute__((aligned(16))) __bf16 smem[];
    typedef Mixed<NK, KF * 32> TK;
    const TK kt{smem}, qt{kt.at + TK::bytes / 2};
    const Mixed<3, C> tt{qt.at + TK::bytes / 2};
    const Mixed<NP, C> mt{tt.at + Mixed<3, C>::bytes / 2};
    float *const sc = reinterpret_cast<float *>(mt.at + Mixed<NP, C>::bytes / 2);

    const uint32_t id = blockIdx.x, h = id / (uint32_t)p.slices % (uint32_t)p.H;
    const int64_t b = id / (uint32_t)p.slices / (uint32_t)p.H;
    const int kh = (int)h / p.each, len = tokens_of(p, b), n = (len + C - 1) / C;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quad = lane >> 4;
    const int64_t head = b * p.H + h, Dv = p.Dv;
    const int c0 = (int)(id % (uint32_t)p.slices) * 64, c = c0 + 16 * wave + l16;
    const bool busy = c0 + 16 * wave < Dv, in = c < Dv;

    f32x4 Z[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dk = 16 * d + 4 * quad + r;
            Z[d][r] = p.dh_last && dk < p.Dk && in ? p.dh_last[(head * p.Dk + dk) * Dv + c] : 0.0f;
        }
    const int64_t mine = h * Dv + min((int64_t)c, Dv - 1);
    ChunkRows<T, KF> kr, qr;
    Square<3> tr;
    Square<NP> mr;
    f32x4 sr;
    ChunkColumn<T> dy;
    auto load = [&](int i, auto full) __attribute__((always_inline)) {
        const int64_t chunk = (b * p.n + i) * p.H + h;
        const int m = min(C, len - i * C);
        kr.template load<full.value, WIDE>(p.k, b, (int64_t)i * C, m, kh, p.Dk);
        qr.template load<full.value, WIDE>(p.q, b, (int64_t)i * C, m, kh, p.Dk);
        tr.load(p.tri, chunk);
        mr.load(p.mix, chunk);
        sr = reinterpret_cast<const f32x4 *>(p.scal + chunk * SCALAR_FLOATS)[tid % (SCALAR_FLOATS / 4)];
    };
    auto load_dy = [&](int i, auto full) __attribute__((always_inline)) {
        dy.template load<full.value>(p.dy, b, (int64_t)i * C, min(C, len - i * C), mine);
    };
    auto scalar = [&](int which, int rt) __attribute__((always_inline)) {
        return *reinterpret_cast<const f32x4 *>(sc + which * C + 16 * rt + 4 * quad);
    };
    // Z += (rows of keys)^T w
    auto into_state = [&](const TK &t, const f32x4 (&w)[RT]) __attribute__((always_inline)) {
        bf16x8 o[2][3];
#pragma unroll
        for (int f = 0; f < 2; ++f) operand<3>(w[2 * f], w[2 * f + 1], o[f]);
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int g = 0; g < DT / 2; ++g) {
                bf16x8 a[2][NK];
                f32x4 two[2] = {Z[2 * g], Z[2 * g + 1]};
                t.cols(f, 2 * g, a[0]);
                t.cols(f, 2 * g + 1, a[1]);
                multiply_rows<3>(two, a, o[f]);
                Z[2 * g] = two[0];
                Z[2 * g + 1] = two[1];
            }
    };

    // Chunk i; `full`: whole, and so is chunk `then`, whose operands go out here
    auto step = [&](int i, int then, auto full) __attribute__((always_inline)) {
        const int64_t t0 = (int64_t)i * C, chunk = (b * p.n + i) * p.H + h;
        const int m = min(C, len - i * C);
        kr.store(kt);
        qr.store(qt);
        tr.store(tt);
        mr.store(mt);
        if (tid < SCALAR_FLOATS / 4) reinterpret_cast<f32x4 *>(sc)[tid] = sr;
        __syncthreads();
        if constexpr (full.value) load(then, full);
        if (busy) {
            put_state<DT>(Z, p.ds + chunk * p.Dk * Dv + c, p.Dk, Dv, in);
            // what reaches u: through the state behind the chunk, and through y
            f32x4 U[RT], W[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) U[rt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int f = 0; f < KF; ++f) {
                bf16x8 z[3], a[RT][NK];
                operand<3>(Z[2 * f], Z[2 * f + 1], z);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) kt.rows(rt, f, a[rt]);
                multiply_rows<3>(U, a, z);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                U[rt] *= scalar(OUT_K, rt);
#pragma unroll
                for (int r = 0; r < 4; ++r) W[rt][r] = (float)dy.v[rt][r];
            }
            if constexpr (full.value) load_dy(then, full);
            {
                bf16x8 y[2][NK], a[RT][NP], au[2][NP];
#pragma unroll
                for (int f = 0; f < 2; ++f) operand<NK>(W[2 * f], W[2 * f + 1], y[f]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) mt.rows(rt, 1, a[rt]);
                multiply_rows<3>(U, a, y[1]);
                f32x4 upper[2] = {U[0], U[1]};
                mt.rows(0, 0, au[0]);
                mt.rows(1, 0, au[1]);
                multiply_rows<3>(upper, au, y[0]);
                U[0] = upper[0];
                U[1] = upper[1];
            }
            const float whole = exp_of(reinterpret_cast<const double *>(sc + SCALARS * C)[C - 1]);
#pragma unroll
            for (int d = 0; d < DT; ++d) Z[d] *= whole;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) W[rt] *= scalar(IN_Q, rt);
            into_state(qt, W);

            f32x4 X[RT];
            {
                bf16x8 u[2][3], a[RT][3], au[2][3];
#pragma unroll
                for (int f = 0; f < 2; ++f) operand<3>(U[2 * f], U[2 * f + 1], u[f]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    X[rt] = f32x4{0, 0, 0, 0};
                    tt.rows(rt, 1, a[rt]);
                }
                multiply_rows<3>(X, a, u[1]);
                f32x4 upper[2] = {X[0], X[1]};
                tt.rows(0, 0, au[0]);
                tt.rows(1, 0, au[1]);
                multiply_rows<3>(upper, au, u[0]);
                X[0] = upper[0];
                X[1] = upper[1];
            }
            put_state<RT>(X, p.dx + chunk * C * Dv + c, C, Dv, in);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                X[rt] *= scalar(BETA, rt);
                W[rt] = -scalar(IN_K, rt) * X[rt];
            }
            put_column<full.value, T>(X, p.dv, b, t0, m, (int)min((int64_t)C, p.L - t0), h * Dv + c, in);
            into_state(kt, W);
        }
        __syncthreads();
    };
    const int whole_chunks = len / C;
    if (whole_chunks < n) {
        load(n - 1, std::false_type());
        load_dy(n - 1, std::false_type());
        step(n - 1, n - 1, std::false_type());
    }
    if (whole_chunks > 0) {
        load(whole_chunks - 1, std::true_type());
        load_dy(whole_chunks - 1, std::true_type());
        for (int i = whole_chunks - 1; i >= 0; --i) step(i, max(i - 1, 0), std::true_type());     // (the first one's again: no branch)
    }
    if (p.dh0) put_state<DT>(Z, p.dh0 + head * p.Dk * Dv + c, p.Dk, Dv, in);
    const int cols = min(64, (int)Dv - c0);
    for (int64_t u = tid; u < (p.L - (int64_t)n * C) * cols; u += NT) {
        const int64_t t = (int64_t)n * C + u / cols;
        static_cast<T *>(p.dv.data)[b * p.dv.s0 + t * p.dv.s1 + h * Dv + c0 + u % cols] = (T)0.0f;
    }
}

// ---------------------------------------------------------------------------
// chunks side by side: the gradients of q, k, g and beta; a workgroup a chunk of a head
// ---------------------------------------------------------------------------
// First the products along v's columns, 32 of them at a time (states, u and x come through LDS in terms); then those along the
// chunk's tokens, for which LDS holds q, k and the matrices of 64 x 64.  A wavefront has 16 tokens' rows of all results.
template <typename T, int KF>
__global__ __launch_bounds__(NT) void merit_delta_grads(DeltaParams p)
{
    constexpr int NK = Terms<T>::n, DT = 2 * KF;
    extern __shared__ __attribute__((aligned(16))) __bf16 smem[];
    __shared__ double G[C], suffix[C], dots[4];
    __shared__ float invk[C], invq[C], beta[C];
    typedef Tile<3, KF * 32, 32> TS;
    typedef Tile<3, C, 32> TU;
    typedef Tile<NK, C, KF * 32> TK;
    typedef Tile<3, C, C> TM;
    const TS st{smem}, zt{st.at + TS::bytes / 2};
    const TU ut{zt.at + TS::bytes / 2};
    const TK kt{smem}, qt{kt.at + TK::bytes / 2};
    const TM pt{qt.at + TK::bytes / 2}, mt{pt.at + TM::bytes / 2};

    const uint32_t id = blockIdx.x, h = id % (uint32_t)p.H, bi = id / (uint32_t)p.H;
    const uint32_t i = bi % (uint32_t)p.n;
    const int64_t b = bi / (uint32_t)p.n, t0 = (int64_t)i * C, Dv = p.Dv;
    const int kh = (int)h / p.each, m = min(C, tokens_of(p, b) - (int)t0), here = min(C, (int)(p.L - t0));
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quad = lane >> 4, row4 = 16 * wave + 4 * quad;
    float *part_q = p.part ? p.part + ((b * p.L + t0) * p.H + h) * p.Dk : nullptr;
    float *part_k = p.part ? part_q + p.B * p.L * p.H * p.Dk : nullptr;
    auto put = [&](int r, int c, float q, float k) __attribute__((always_inline)) {
        if (p.part) {
            part_q[(int64_t)r * p.H * p.Dk + c] = q;
            part_k[(int64_t)r * p.H * p.Dk + c] = k;
        } else {
            static_cast<T *>(p.dq.data)[b * p.dq.s0 + (t0 + r) * p.dq.s1 + (int64_t)kh * p.Dk + c] = (T)q;
            static_cast<T *>(p.dk.data)[b * p.dk.s0 + (t0 + r) * p.dk.s1 + (int64_t)kh * p.Dk + c] = (T)k;
        }
    };
    auto put_gates = [&](int r, float dg, float db) __attribute__((always_inline)) {
        if (p.dg.data) static_cast<float *>(p.dg.data)[b * p.dg.s0 + (t0 + r) * p.dg.s1 + h] = dg;
        static_cast<float *>(p.dbeta.data)[b * p.dbeta.s0 + (t0 + r) * p.dbeta.s1 + h] = db;
    };
    if (m <= 0) {
        for (int u = tid; u < here * p.Dk; u += NT) put(u / p.Dk, u % p.Dk, 0.0f, 0.0f);
        if (tid < here) put_gates(tid, 0.0f, 0.0f);
        return;
    }
    const float *scal = p.scal + (int64_t)id * SCALAR_FLOATS;
    if (tid < C) {
        G[tid] = reinterpret_cast<const double *>(scal + SCALARS * C)[tid];
        invk[tid] = scal[INV_K * C + tid];
        invq[tid] = scal[INV_Q * C + tid];
        beta[tid] = scal[BETA * C + tid];
    }
    const float *state = p.states + (int64_t)id * (p.Dk + C) * Dv, *kept = state + p.Dk * Dv;
    const float *z = p.ds + (int64_t)id * p.Dk * Dv, *x = p.dx + (int64_t)id * C * Dv;
    const int own = 16 * wave + l16;
    const float bt = scal[BETA * C + own];
    const T *dyrow = static_cast<const T *>(p.dy.data) + b * p.dy.s0 + (t0 + own) * p.dy.s1 + h * Dv;

    f32x4 dq[DT], rows[DT], cols[DT], dP[4], dM[4];
#pragma unroll
    for (int d = 0; d < DT; ++d) dq[d] = rows[d] = cols[d] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) dP[j] = dM[j] = f32x4{0, 0, 0, 0};
    float db = 0.0f;
    double sz = 0.0;
    for (int c0 = 0; c0 < Dv; c0 += 32) {
        __syncthreads();
        float szp = 0.0f;
        for (int u = tid; u < KF * 32 * 4; u += NT) {
            const int r = u / 4, c = u % 4 * 8;
            Eight<float> s = zero8<float>(), g = zero8<float>();
            if (r < p.Dk) {
                s = load8<float>(state + r * Dv + c0, c, p.Dv - c0, p.wide_v);
                g = load8<float>(z + r * Dv + c0, c, p.Dv - c0, p.wide_v);
            }
            bf16x8 o[3];
            terms8<float>(s, o);
            st.put8(r, c, o);
            terms8<float>(g, o);
            zt.put8(r, c, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) szp = fmaf(s.v[e], g.v[e], szp);
        }
        sz += (double)szp;
        {
            const int r = tid / 4, c = tid % 4 * 8;
            Eight<float> d = load8<float>(kept + r * Dv + c0, c, p.Dv - c0, p.wide_v);
            const float f = scal[BETA * C + r];
#pragma unroll
            for (int e = 0; e < 8; ++e) d.v[e] *= f;
            bf16x8 o[3];
            terms8<float>(d, o);
            ut.put8(r, c, o);
        }
        bf16x8 ya[NK], xa[3], ua[3];
        {
            Eight<T> y = zero8<T>();
            if (own < m) y = load8<T>(dyrow + c0, 8 * quad, p.Dv - c0, p.wide_v);
            terms8<T>(y, ya);
            const Eight<float> xe = load8<float>(x + own * Dv + c0, 8 * quad, p.Dv - c0, p.wide_v);
            const Eight<float> d = load8<float>(kept + own * Dv + c0, 8 * quad, p.Dv - c0, p.wide_v);
            terms8<float>(xe, xa);
#pragma unroll
            for (int e = 0; e < 8; ++e) db = fmaf(xe.v[e], d.v[e], db);
        }
        __syncthreads();
        ut.rows(16 * wave, 0, ua);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            bf16x8 o[3];
            st.rows(16 * d, 0, o);
            multiply<3>(dq[d], ya, o);
            multiply<3>(rows[d], xa, o);
            zt.rows(16 * d, 0, o);
            multiply<3>(cols[d], ua, o);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j > wave) continue;
            bf16x8 o[3];
            ut.rows(16 * j, 0, o);
            multiply<3>(dP[j], ya, o);
            multiply<3>(dM[j], xa, o);
        }
    }
    (void)bt;
    db += lane_xor<4>(db);
    db += lane_xor<5>(db);
#pragma unroll
    for (int s = 1; s < 64; s *= 2) sz += __shfl_xor(sz, s);
    if (lane == 0) dots[wave] = sz;

    // scales of rows; K and Q; the matrices of 64 x 64, rows side by side
    float in[4], out[4], ik[4], iq[4], bb[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const double g = G[row4 + r];
        in[r] = exp_of(g);
        out[r] = exp_of(G[C - 1] - g);
        ik[r] = invk[row4 + r];
        iq[r] = invq[row4 + r];
        bb[r] = beta[row4 + r];
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            dq[d][r] *= in[r];
            rows[d][r] *= -in[r] * bb[r];
            cols[d][r] *= out[r];
        }
    __syncthreads();            // (the first part's LDS is free)
    {
        ChunkRows<T, KF> e;
        if (p.wide_qk) e.template load<false, true>(p.k, b, t0, m, kh, p.Dk);
        else e.template load<false, false>(p.k, b, t0, m, kh, p.Dk);
        e.store(kt);
        if (p.wide_qk) e.template load<false, true>(p.q, b, t0, m, kh, p.Dk);
        else e.template load<false, false>(p.q, b, t0, m, kh, p.Dk);
        e.store(qt);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j > (wave | 1)) continue;
        const int c = 16 * j + l16;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = row4 + r;
            const float f = c <= t ? exp_of(G[t] - G[c]) : 0.0f;
            dP[j][r] = c <= t ? f * dP[j][r] : 0.0f;
            dM[j][r] = c < t ? -f * bb[r] * dM[j][r] : 0.0f;
            pt.put1(t, c, dP[j][r] * invk[c]);
            mt.put1(t, c, dM[j][r] * invk[c]);
        }
    }
    __syncthreads();
    // K.(o u Z^T), for the last token's G
    float kz = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) kz = fmaf(ik[r] * kt.value(row4 + r, 16 * d + l16), cols[d][r], kz);
    double kzd = (double)kz;
#pragma unroll
    for (int s = 1; s < 64; s *= 2) kzd += __shfl_xor(kzd, s);
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        if (2 * f > wave) continue;
        bf16x8 pa[3], ma[3];
        pt.rows(16 * wave, 32 * f, pa);
        mt.rows(16 * wave, 32 * f, ma);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            bf16x8 o[NK];
            kt.cols(32 * f, 16 * d, o);
            multiply<3>(dq[d], pa, o);
            multiply<3>(rows[d], ma, o);
        }
    }
    __syncthreads();
    // their transposes
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (j > (wave | 1)) continue;
        float e[4], g[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            e[r] = dP[j][r] * iq[r] * p.scale;
            g[r] = dM[j][r] * ik[r];
        }
        pt.put4(16 * j + l16, row4, e);
        mt.put4(16 * j + l16, row4, g);
    }
    __syncthreads();
#pragma unroll
    for (int f = 0; f < 2; ++f) {
        if (2 * f + 1 < wave) continue;
        bf16x8 pa[3], ma[3];
        pt.rows(16 * wave, 32 * f, pa);
        mt.rows(16 * wave, 32 * f, ma);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            bf16x8 o[NK];
            qt.cols(32 * f, 16 * d, o);
            multiply<3>(cols[d], pa, o);
            kt.cols(32 * f, 16 * d, o);
            multiply<3>(cols[d], ma, o);
        }
    }
    // dots of a row along the keys, through the length, results
    float dotq[4], dotr[4], dotc[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) dotq[r] = dotr[r] = dotc[r] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float kv = kt.value(row4 + r, 16 * d + l16), qv = qt.value(row4 + r, 16 * d + l16);
            dotq[r] = fmaf(qv, dq[d][r], dotq[r]);
            dotr[r] = fmaf(kv, rows[d][r], dotr[r]);
            dotc[r] = fmaf(kv, cols[d][r], dotc[r]);
        }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        dotq[r] = sum_lanes(dotq[r], 16) * iq[r] * p.scale;
        dotr[r] = sum_lanes(dotr[r], 16) * ik[r];
        dotc[r] = sum_lanes(dotc[r], 16) * ik[r];
        if (l16 == 0) suffix[row4 + r] = (double)dotq[r] + (double)dotr[r] - (double)dotc[r];
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int c = 16 * d + l16;
            if (row4 + r >= here || c >= p.Dk) continue;
            float q = dq[d][r] * p.scale, k = rows[d][r] + cols[d][r];
            if (p.unit) {
                q = iq[r] * (q - iq[r] * qt.value(row4 + r, c) * dotq[r]);
                k = ik[r] * (k - ik[r] * kt.value(row4 + r, c) * (dotr[r] + dotc[r]));
            }
            const bool live = row4 + r < m;
            put(row4 + r, c, live ? q : 0.0f, live ? k : 0.0f);
        }
    __shared__ double last[4];
    if (lane == 0) last[wave] = kzd;
    __syncthreads();
    if (wave == 0) {
        double s = suffix[lane];
        if (lane == C - 1)
            s += (double)exp_of(G[C - 1]) * ((dots[0] + dots[1]) + (dots[2] + dots[3])) + (last[0] + last[1]) + (last[2] + last[3]);
#pragma unroll
        for (int k = 1; k < C; k *= 2) {
            const double o = __shfl_down(s, k);
            if (lane + k < C) s += o;
        }
        if (lane < here && p.dg.data)
            static_cast<float *>(p.dg.data)[b * p.dg.s0 + (t0 + lane) * p.dg.s1 + h] = lane < m ? (float)s : 0.0f;
    }
    if (quad == 0 && own < here)
        static_cast<float *>(p.dbeta.data)[b * p.dbeta.s0 + (t0 + own) * p.dbeta.s1 + h] = own < m ? db : 0.0f;
}

// dq, dk of a key head: the sum over its value heads
template <typename T> __global__ __launch_bounds__(NT) void merit_delta_sum_heads(DeltaParams p)
{
    const int64_t u = (int64_t)blockIdx.x * NT + threadIdx.x, row = (int64_t)p.K * p.Dk;
    if (u >= p.B * p.L * row) return;
    const int64_t bt = u / row;
    const int kh = (int)(u % row / p.Dk), c = (int)(u % p.Dk);
    const float *in = p.part + (bt * p.H + (int64_t)kh * p.each) * p.Dk + c;
    float q = 0.0f, k = 0.0f;
    for (int e = 0; e < p.each; ++e) {
        q += in[(int64_t)e * p.Dk];
        k += in[(int64_t)e * p.Dk + p.B * p.L * p.H * p.Dk];
    }
    const int64_t b = bt / p.L, t = bt % p.L;
    static_cast<T *>(p.dq.data)[b * p.dq.s0 + t * p.dq.s1 + (int64_t)kh * p.Dk + c] = (T)q;
    static_cast<T *>(p.dk.data)[b * p.dk.s0 + t * p.dk.s1 + (int64_t)kh * p.Dk + c] = (T)k;
}

template <typename T, int KF> hipError_t backward_chunks(DeltaParams p, hipStream_t s)
{
    constexpr int lds = 2 * Mixed<Terms<T>::n, KF * 32>::bytes + Mixed<3, C>::bytes + Mixed<mix_terms<T>(true), C>::bytes + SCALAR_FLOATS * 4;
    static_assert(lds <= 160 * 1024, "");
    p.slices = (p.Dv + 63) / 64;
    const unsigned grid = (unsigned)(p.B * p.H * p.slices);
    if (p.wide_qk) merit_delta_back_chunks<T, KF, true><<<grid, NT, lds, s>>>(p);
    else merit_delta_back_chunks<T, KF, false><<<grid, NT, lds, s>>>(p);
    return hipGetLastError();
}
template <typename T, int KF> hipError_t grads_of(const DeltaParams &p, hipStream_t s)
{
    constexpr int NK = Terms<T>::n;
    constexpr int one = 2 * Tile<3, KF * 32, 32>::bytes + Tile<3, C, 32>::bytes;
    constexpr int two = 2 * Tile<NK, C, KF * 32>::bytes + 2 * Tile<3, C, C>::bytes;
    constexpr int lds = one > two ? one : two;
    static_assert(lds + 3 * 1024 <= 160 * 1024, "");
    merit_delta_grads<T, KF><<<(unsigned)(p.B * p.n * p.H), NT, lds, s>>>(p);
    return hipGetLastError();
}
template <typename T, int KF> hipError_t backward_of(const DeltaParams &p, hipStream_t s)
{
    if (hipError_t e = prepare_of<T, KF, true>(p, s)) return e;
    if (hipError_t e = backward_chunks<T, KF>(p, s)) return e;
    if (p.n == 0) return hipSuccess;
    if (hipError_t e = grads_of<T, KF>(p, s)) return e;
    if (!p.part) return hipSuccess;
    const int64_t values = p.B * p.L * p.K * p.Dk;
    merit_delta_sum_heads<T><<<(unsigned)((values + NT - 1) / NT), NT, 0, s>>>(p);
    return hipGetLastError();
}
template <typename T> hipError_t backward_typed(const DeltaParams &p, hipStream_t s)
{
    return p.Dk <= 32 ? backward_of<T, 1>(p, s) : p.Dk <= 64 ? backward_of<T, 2>(p, s) : backward_of<T, 4>(p, s);
}

// The passes of one type, each in a file of its own (delta_*.hip)
enum { FORWARD, BACKWARD, STEP };
template <typename T> hipError_t passes(const DeltaParams &p, int pass, hipStream_t s)
{
    if (pass == FORWARD) return forward_typed<T>(p, s);
    return pass == STEP ? token_typed<T>(p, s) : backward_typed<T>(p, s);
}
hipError_t passes_f32(const DeltaParams &p, int pass, hipStream_t s);
hipError_t passes_f16(const DeltaParams &p, int pass, hipStream_t s);
hipError_t passes_bf16(const DeltaParams &p, int pass, hipStream_t s);

}  // namespace delta
}  // namespace merit
