// The gated delta rule, forward: what a chunk's tokens do to each other (merit_delta_prepare), chunk after chunk
// (merit_delta_chunks), one token (merit_delta_token).  The formulas stand in delta.h.
#pragma once

#include "delta.h"

namespace merit {
namespace delta {

// ---------------------------------------------------------------------------
// chunks side by side: a workgroup a chunk of a head
// ---------------------------------------------------------------------------
// It leaves -W and P in terms, their columns interleaved, and the tokens' factors.
template <typename T, int KF, bool WIDE>
__global__ __launch_bounds__(NT) void merit_delta_prepare(DeltaParams p)
{
    constexpr int NK = Terms<T>::n, LINE = C + 4;
    // K, and where it is not needed any more W
    constexpr int first = Tile<NK, C, KF * 32>::bytes > C * LINE * 4 ? Tile<NK, C, KF * 32>::bytes : C * LINE * 4;
    __shared__ __attribute__((aligned(16))) __bf16 kmem[first / 2];
    __shared__ __attribute__((aligned(16))) float a[C][LINE];
    float (*const x)[LINE] = reinterpret_cast<float (*)[LINE]>(kmem);
    __shared__ double G[C];
    __shared__ __attribute__((aligned(16))) float beta[C], finite_beta[C], invk[C], invq[C];
    __shared__ int bad;             // the first token whose row of N is not finite
    const Tile<NK, C, KF * 32> kt{kmem};

    const uint32_t id = blockIdx.x, h = id % (uint32_t)p.H, bi = id / (uint32_t)p.H;
    const uint32_t i = bi % (uint32_t)p.n;
    const int64_t b = bi / (uint32_t)p.n, t0 = (int64_t)i * C;
    const int kh = (int)h / p.each, m = min(C, tokens_of(p, b) - (int)t0);
    if (m <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quad = lane >> 4;
    const Prepared to = prepared(p, id);
    float *const scal = to.scal;

    // Two rows' loads in a wavefront: keys to LDS, their squares' sums over the lanes of a row
    ChunkRows<T, KF> kr;
    kr.template load<false, WIDE>(p.k, b, t0, m, kh, p.Dk);
    const int own = 16 * wave + l16;
    const T *qrow = static_cast<const T *>(p.q.data) + b * p.q.s0 + (t0 + min(own, m - 1)) * p.q.s1 + (int64_t)kh * p.Dk;
    Eight<T> qe[KF];
#pragma unroll
    for (int f = 0; f < KF; ++f) qe[f] = take8<WIDE, T>(qrow, 32 * f + 8 * quad, own < m ? p.Dk : 0);
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
        finite_beta[lane] = isfinite(bt) ? bt : 0.0f;     // (the rows that it reaches are lost anyway)
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

    // Rows 16 wave .. of K K^T and Q K^T, transposed (the lane then has four values of a row side by side), up to the diagonal's block
    bf16x8 qa[KF][NK], ka[KF][NK];
#pragma unroll
    for (int f = 0; f < KF; ++f) {
        terms8<T>(qe[f], qa[f]);
        kt.rows(16 * wave, 32 * f, ka[f]);
    }
    const int t = own;                                  // the token that reads
    const double gt = G[t];
    const float kt_len = invk[t], qt_len = invq[t] * p.scale;
#pragma unroll
    for (int jb = 0; jb < 4; ++jb) {
        f32x4 kk = {0, 0, 0, 0}, qk = {0, 0, 0, 0};
        if (jb <= wave)
#pragma unroll
            for (int f = 0; f < KF; ++f) {
                bf16x8 o[NK];
                kt.rows(16 * jb, 32 * f, o);
                multiply<3>(kk, o, ka[f]);
                multiply<3>(qk, o, qa[f]);
            }
        const int j0 = 16 * jb + 4 * quad;              // the tokens that were written
        const f32x4 lens = *reinterpret_cast<const f32x4 *>(&invk[j0]);
        f32x4 n;
        bf16x4 out[3];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = j0 + r;
            const float f = j <= t ? exp_of(gt - G[j]) * lens[r] : 0.0f;
            float w = j < t ? f * kt_len * kk[r] : 0.0f;
            if (j < t && !isfinite(w * beta[j])) {      // (0 times it would reach the tokens before)
                atomicMin(&bad, t);
                w = 0.0f;
            }
            n[r] = w;
            __bf16 s[3];
            split<3>(j <= t ? f * qt_len * qk[r] : 0.0f, s);
#pragma unroll
            for (int k = 0; k < 3; ++k) out[k][r] = s[k];
        }
        *reinterpret_cast<f32x4 *>(&a[t][j0]) = n;
        if (jb <= (wave | 1))
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (k < p.mix_terms) *reinterpret_cast<bf16x4 *>(to.mix + k * TRIANGLE + triangle_at(t, interleaved(j0))) = out[k];
    }
    __syncthreads();

    // W in blocks of 16 x 16.  On the diagonal: lane c of wavefront w has column c of block w and takes one row after the other,
    // W_rc = N_rc - sum over c < j < r of N_rj b_j W_jc (powers of a block, which would do it with products, cancel where keys are
    // alike).
    {
        float d[16];                // b W
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float v0 = a[16 * wave + r][16 * wave + l16], v1 = 0.0f;        // (0 from the diagonal on)
#pragma unroll
            for (int j = 0; j < r; j += 4) {
                const f32x4 w = *reinterpret_cast<const f32x4 *>(&a[16 * wave + r][16 * wave + j]);
                v0 = fmaf(-w[0], d[j], v0);
                if (j + 1 < r) v1 = fmaf(-w[1], d[j + 1], v1);
                if (j + 2 < r) v0 = fmaf(-w[2], d[j + 2], v0);
                if (j + 3 < r) v1 = fmaf(-w[3], d[j + 3], v1);
            }
            const float v = v0 + v1;
            d[r] = finite_beta[16 * wave + r] * v;
            if (quad == 0) x[16 * wave + r][16 * wave + l16] = v;
        }
    }
    __syncthreads();
    // Below it, a diagonal of blocks at a time: W_ij = M - W_ii (b M), M = N_ij - N_ij (b W_jj) - .. - N_i,i-1 (b W_i-1,j), fp32
    // products.  Step s of a product sums over the numbers 4 q + s of quad q's lanes, which is how a result lies in them: it goes
    // on without a move.
#pragma unroll
    for (int dist = 1; dist < 4; ++dist) {
        const int bi_ = wave + dist, bj = wave;
        if (bi_ < 4) {
            f32x4 mm;
#pragma unroll
            for (int r = 0; r < 4; ++r) mm[r] = a[16 * bi_ + 4 * quad + r][16 * bj + l16];
#pragma unroll
            for (int k = 0; k < dist; ++k) {
                const f32x4 bk = *reinterpret_cast<const f32x4 *>(&finite_beta[16 * (bj + k) + 4 * quad]);
                const f32x4 ak = *reinterpret_cast<const f32x4 *>(&a[16 * bi_ + l16][16 * (bj + k) + 4 * quad]);
#pragma unroll
                for (int s = 0; s < 4; ++s)
                    mm = __builtin_amdgcn_mfma_f32_16x16x4f32(-ak[s], bk[s] * x[16 * (bj + k) + 4 * quad + s][16 * bj + l16], mm, 0, 0, 0);
            }
            const f32x4 bm = *reinterpret_cast<const f32x4 *>(&finite_beta[16 * bi_ + 4 * quad]) * mm;
            const f32x4 wi = *reinterpret_cast<const f32x4 *>(&x[16 * bi_ + l16][16 * bi_ + 4 * quad]);
#pragma unroll
            for (int s = 0; s < 4; ++s) mm = __builtin_amdgcn_mfma_f32_16x16x4f32(-wi[s], bm[s], mm, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[16 * bi_ + 4 * quad + r][16 * bj + l16] = mm[r];
        }
        __syncthreads();
    }
    // -W in three terms, zeros above the diagonal's blocks: a thread has 16 values of a row
    {
        const int r = tid >> 2, c0 = 16 * (tid & 3);
        if (r < C / 2 && c0 >= C / 2) return;
        const bool lost = r >= bad, below = r >> 4 >= c0 >> 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(&x[r][c0 + 4 * k]);
            bf16x4 o[3];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                __bf16 s[3];
                split<3>(lost ? __builtin_nanf("") : below ? -v[e] : 0.0f, s);
#pragma unroll
                for (int n = 0; n < 3; ++n) o[n][e] = s[n];
            }
#pragma unroll
            for (int n = 0; n < 3; ++n) *reinterpret_cast<bf16x4 *>(to.w + n * TRIANGLE + triangle_at(r, interleaved(c0 + 4 * k))) = o[n];
        }
    }
}

// ---------------------------------------------------------------------------
// one chunk after the other: a wavefront 16 columns of a head's state
// ---------------------------------------------------------------------------
// The columns of a state do not depend on each other.  A wavefront has 16 of them, all of a chunk's tokens and all rows of the state,
// in registers: results go from product to product as they lie (delta.h: Mixed).  LDS holds the other operands, K, Q and the two
// triangular matrices, for the four wavefronts of a workgroup; the next chunk's are on their way in registers meanwhile.
template <typename T, int KF, bool WIDE>
__global__ __launch_bounds__(NT) void merit_delta_chunks(DeltaParams p)
{
    constexpr int NK = Terms<T>::n, NP = mix_terms<T>(), ORD = NP, RT = C / 16, DT = 2 * KF;
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
    const bool busy = c0 + 16 * wave < Dv, in = c < Dv;            // (the wavefront, the lane has columns)

    f32x4 S[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dk = 16 * d + 4 * quad + r;
            S[d][r] = p.h0 && dk < p.Dk && in ? p.h0[(head * p.Dk + dk) * Dv + c] : 0.0f;
        }
    const int64_t mine = h * Dv + min((int64_t)c, Dv - 1);         // (a lane without a column: any that is there)
    ChunkRows<T, KF> kr, qr;
    Triangle<3> tr;
    Triangle<NP> mr;
    f32x4 sr;
    ChunkColumn<T> v;
    auto load = [&](int i, auto full) __attribute__((always_inline)) {
        const int64_t chunk = (b * p.n + i) * p.H + h;
        const int m = min(C, len - i * C);
        kr.template load<full.value, WIDE>(p.k, b, (int64_t)i * C, m, kh, p.Dk);
        qr.template load<full.value, WIDE>(p.q, b, (int64_t)i * C, m, kh, p.Dk);
        const Prepared from = prepared(p, chunk);
        tr.load(from.w);
        mr.load(from.mix);
        sr = reinterpret_cast<const f32x4 *>(from.scal)[tid % (SCALAR_FLOATS / 4)];
    };
    auto load_v = [&](int i, auto full) __attribute__((always_inline)) {
        v.template load<full.value>(p.v, b, (int64_t)i * C, min(C, len - i * C), mine);
    };
    auto scalar = [&](int which, int rt) __attribute__((always_inline)) {
        return *reinterpret_cast<const f32x4 *>(sc + which * C + 16 * rt + 4 * quad);
    };
    // Values that are not finite go into products as zeros, because those of earlier tokens have them too, times 0; `bad` is the
    // first token of the chunk from which the lane's column has some, and everything from there on becomes a NaN.
    int bad = C;
    auto finite = [&](f32x4 (&x)[RT]) __attribute__((always_inline)) {
        bool all = true;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) all = all && isfinite(x[rt][r]);
        if (__ballot(!all) == 0) return;
#pragma unroll
        for (int rt = RT - 1; rt >= 0; --rt)
#pragma unroll
            for (int r = 3; r >= 0; --r)
                if (!isfinite(x[rt][r])) {
                    bad = min(bad, 16 * rt + 4 * quad + r);
                    x[rt][r] = 0.0f;
                }
        bad = min(bad, __shfl_xor(bad, 16));
        bad = min(bad, __shfl_xor(bad, 32));
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
            // K S and Q S
            f32x4 X[RT], Y[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) X[rt] = Y[rt] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int f = 0; f < KF; ++f) {
                bf16x8 s[3], a[RT][NK];
                operand<3>(S[2 * f], S[2 * f + 1], s);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) kt.rows(rt, f, a[rt]);
                multiply_rows<3>(X, a, s);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) qt.rows(rt, f, a[rt]);
                multiply_rows<ORD>(Y, a, s);
            }
            if (p.states) put_state<DT>(S, p.states + chunk * p.prep_stride + PREPARED_FLOATS + c, p.Dk, Dv, in);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const f32x4 in_k = scalar(IN_K, rt);
#pragma unroll
                for (int r = 0; r < 4; ++r) X[rt][r] = fmaf(-in_k[r], X[rt][r], (float)v.v[rt][r]);
            }
            if constexpr (full.value) load_v(then, full);

            // d, u
            f32x4 D[RT], U[RT];
            bf16x8 x[2][3];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                D[rt] = X[rt];
                X[rt] *= scalar(BETA, rt);
            }
            finite(X);
#pragma unroll
            for (int f = 0; f < 2; ++f) operand<3>(X[2 * f], X[2 * f + 1], x[f]);
            {
                bf16x8 a[RT][3];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) tt.rows(rt, 0, a[rt]);
                multiply_rows<3>(D, a, x[0]);
                f32x4 lower[2] = {D[2], D[3]};
                bf16x8 al[2][3];
                tt.rows(2, 1, al[0]);
                tt.rows(3, 1, al[1]);
                multiply_rows<3>(lower, al, x[1]);
                D[2] = lower[0];
                D[3] = lower[1];
            }
            if (__ballot(bad < C) != 0)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * rt + 4 * quad + r >= bad) D[rt][r] = __builtin_nanf("");
            if (p.states) {
                put_state<RT>(D, p.states + chunk * p.prep_stride + PREPARED_FLOATS + p.Dk * Dv + c, C, Dv, in);
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) U[rt] = D[rt] * scalar(BETA, rt);
            finite(U);

            // the state behind the chunk
            const float whole = exp_of(reinterpret_cast<const double *>(sc + SCALARS * C)[C - 1]);
            {
                bf16x8 o[2][3];
                f32x4 w[RT];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) w[rt] = U[rt] * scalar(OUT_K, rt);
#pragma unroll
                for (int f = 0; f < 2; ++f) operand<3>(w[2 * f], w[2 * f + 1], o[f]);
#pragma unroll
                for (int d = 0; d < DT; ++d) S[d] *= whole;
#pragma unroll
                for (int f = 0; f < 2; ++f)
#pragma unroll
                    for (int g = 0; g < DT / 2; ++g) {
                        bf16x8 a[2][NK];
                        f32x4 two[2] = {S[2 * g], S[2 * g + 1]};
                        kt.cols(f, 2 * g, a[0]);
                        kt.cols(f, 2 * g + 1, a[1]);
                        multiply_rows<3>(two, a, o[f]);
                        S[2 * g] = two[0];
                        S[2 * g + 1] = two[1];
                    }
            }
            // y
            {
                bf16x8 u[2][NP], a[RT][NP], al[2][NP];
#pragma unroll
                for (int f = 0; f < 2; ++f) operand<NP>(U[2 * f], U[2 * f + 1], u[f]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    Y[rt] *= scalar(IN_Q, rt);
                    mt.rows(rt, 0, a[rt]);
                }
                multiply_rows<ORD>(Y, a, u[0]);
                f32x4 lower[2] = {Y[2], Y[3]};
                mt.rows(2, 1, al[0]);
                mt.rows(3, 1, al[1]);
                multiply_rows<ORD>(lower, al, u[1]);
                Y[2] = lower[0];
                Y[3] = lower[1];
            }
            if (__ballot(bad < C) != 0 && bad < C) {
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * rt + 4 * quad + r >= bad) Y[rt][r] = __builtin_nanf("");
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[d][r] = __builtin_nanf("");
            }
            put_column<full.value, T>(Y, p.y, b, t0, m, (int)min((int64_t)C, p.L - t0), h * Dv + c, in);
        }
        __syncthreads();
    };
    const int whole_chunks = len / C;
    if (whole_chunks > 0) {
        load(0, std::true_type());
        load_v(0, std::true_type());
        for (int i = 0; i < whole_chunks; ++i) step(i, min(i + 1, whole_chunks - 1), std::true_type());    // (the last one's again: no branch)
    }
    if (whole_chunks < n) {
        load(n - 1, std::false_type());
        load_v(n - 1, std::false_type());
        step(n - 1, n - 1, std::false_type());
    }
    if (p.h_last) put_state<DT>(S, p.h_last + head * p.Dk * Dv + c, p.Dk, Dv, in);
    // zeros behind the sequence's last chunk
    const int cols = min(64, (int)Dv - c0);
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

template <typename T, int KF> hipError_t prepare_of(const DeltaParams &p, hipStream_t s)
{
    const unsigned grid = (unsigned)(p.B * p.n * p.H);
    if (grid == 0) return hipSuccess;
    if (p.wide_qk) merit_delta_prepare<T, KF, true><<<grid, NT, 0, s>>>(p);
    else merit_delta_prepare<T, KF, false><<<grid, NT, 0, s>>>(p);
    return hipGetLastError();
}
template <typename T, int KF> hipError_t forward_of(DeltaParams p, hipStream_t s)
{
    constexpr int lds = 2 * Mixed<Terms<T>::n, KF * 32>::bytes + Mixed<3, C>::bytes + Mixed<mix_terms<T>(), C>::bytes + SCALAR_FLOATS * 4;
    static_assert(lds <= 160 * 1024, "");
    p.mix_terms = p.states ? 3 : mix_terms<T>();
    if (hipError_t e = prepare_of<T, KF>(p, s)) return e;
    p.slices = (p.Dv + 63) / 64;
    const unsigned grid = (unsigned)(p.B * p.H * p.slices);
    if (p.wide_qk) merit_delta_chunks<T, KF, true><<<grid, NT, lds, s>>>(p);
    else merit_delta_chunks<T, KF, false><<<grid, NT, lds, s>>>(p);
    return hipGetLastError();
}
template <typename T> hipError_t forward_typed(const DeltaParams &p, hipStream_t s)
{
    return p.Dk <= 32 ? forward_of<T, 1>(p, s) : p.Dk <= 64 ? forward_of<T, 2>(p, s) : forward_of<T, 4>(p, s);
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
