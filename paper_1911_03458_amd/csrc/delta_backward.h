// The gated delta rule, backward (the formulas and the representation of operands: delta.h).  With Z the gradient of the state
// behind a chunk, K and Q of unit length (Q scaled), i = exp(G), o = exp(G_C - G):
//     y = P^T dy + o K Z,   x = y - W^T (b y),   dv = b x,   Z_before = exp(G_C) Z + Q^T (i dy) - K^T (i dv)              one chunk after the other
//     dQ = i (dy S_0^T) + (f o dy u^T) K                                                                   chunks side by side
//     dK = rows + cols,  rows = M K - i (dv S_0^T),  cols = (f o dy u^T)^T Q + M^T K + o (u Z^T),  M = -b f o (x u^T) below the diagonal
//     db = x.d,   dG = Q.dQ + K.rows - K.cols, at the last token besides exp(G_C) <S_0, Z> + K.(o u Z^T),   dg_t = sum of dG from t on
// d, S_0, W and P come from the forward pass.
#pragma once

#include "delta_forward.h"

namespace merit {
namespace delta {

// ---------------------------------------------------------------------------
// one chunk after the other, from the last: two wavefronts 16 columns of a head's Z
// ---------------------------------------------------------------------------
// Split and bound as merit_delta_chunks is; here the second half's tokens come first.  The triangular matrices' transposes come out
// of transposing reads.  128 heads of 2048 tokens, states of 128 x 128, bfloat16: 277 us (0.79 GB, 2.9 TB/s), of which about 15 are
// for keeping values that are not finite away from later tokens.
template <typename T, int KF> struct BackwardLds {
    static constexpr int NK = Terms<T>::n;
    static constexpr int k = 0, w = k + Keys<NK, KF * 32>::bytes, mix = w + Triangle<3>::bytes, scal = mix + Triangle<3>::bytes,
                         q = scal + SCALAR_FLOATS * 4;
    // handed over in a pair: 2 KB to each, b y of the second and then w of the first, w of the second
    static constexpr bool shared = NK == 3 && KF == 4;
    static constexpr int pair = (4 + 3 + 3) * 1024, hand = shared ? q : q + Keys<NK, KF * 32>::bytes;
    static constexpr int bytes = hand + 4 * pair > q + Keys<NK, KF * 32>::bytes ? hand + 4 * pair : q + Keys<NK, KF * 32>::bytes;
};
// (a half at a time is compiled: every place in LDS is then a lane's base and a constant)
template <typename T, int KF, bool WIDE, int half>
__device__ __forceinline__ void backward_half(const DeltaParams &p, __bf16 *smem, int *lost)
{
    typedef BackwardLds<T, KF> L;
    constexpr int NK = L::NK, KO = KF < 2 ? 1 : KF / 2;
    char *const lds = reinterpret_cast<char *>(smem);
    const Keys<NK, KF * 32> kt{reinterpret_cast<__bf16 *>(lds + L::k)}, qt{reinterpret_cast<__bf16 *>(lds + L::q)};
    const Triangle<3> wt{reinterpret_cast<__bf16 *>(lds + L::w)}, mt{reinterpret_cast<__bf16 *>(lds + L::mix)};
    float *const sc = reinterpret_cast<float *>(lds + L::scal);

    const uint32_t id = blockIdx.x, h = id / (uint32_t)p.slices % (uint32_t)p.H;
    const int64_t b = id / (uint32_t)p.slices / (uint32_t)p.H;
    const int kh = (int)h / p.each, len = tokens_of(p, b), n = (len + C - 1) / C;
    const int tid = threadIdx.x, lane = tid & 63, tile = __builtin_amdgcn_readfirstlane(tid >> 6 & 3), l16 = lane & 15, quad = lane >> 4;
    const int64_t head = b * p.H + h, Dv = p.Dv;
    const int c0 = (int)(id % (uint32_t)p.slices) * p.width, c = c0 + 16 * tile + l16;
    const bool busy = 16 * tile < p.width && c0 + 16 * tile < Dv, in = busy && c < Dv, has = half < KF;
    f32x4 *const to_me = reinterpret_cast<f32x4 *>(lds + L::hand + tile * L::pair + half * 2048) + lane;
    f32x4 *const to_other = reinterpret_cast<f32x4 *>(lds + L::hand + tile * L::pair + (1 - half) * 2048) + lane;
    bf16x8 *const one = reinterpret_cast<bf16x8 *>(lds + L::hand + tile * L::pair + 4096) + lane;     // b y of the second, w of the first
    bf16x8 *const two = one + 192;                                                                       // w of the second

    f32x4 Z[KO][2];
#pragma unroll
    for (int o = 0; o < KO; ++o) {
        const int dk = 32 * (half + 2 * o);
        get_rows(Z[o], p.dh_last ? p.dh_last + (head * p.Dk + dk) * Dv + c : nullptr, p.Dk - dk, Dv, in);
    }
    const int64_t mine = h * Dv + min((int64_t)c, Dv - 1);
    // (the second half's wavefronts, which wait for the others later, move what the next chunk needs)
    ChunkRows<T, KF, NT> kr, qr;
    TriangleRows<3, NT> wr, mr;
    f32x4 sr;
    ChunkColumn<T, 2> dy;
    auto load = [&](int i, auto full) __attribute__((always_inline)) {
        const int m = min(C, len - i * C);
        kr.template load<full.value, WIDE>(p.k, b, (int64_t)i * C, m, kh, p.Dk);
        qr.template load<full.value, WIDE>(p.q, b, (int64_t)i * C, m, kh, p.Dk);
        const Prepared from = prepared(p, (b * p.n + i) * p.H + h);
        wr.load(from.w);
        mr.load(from.mix);
        sr = reinterpret_cast<const f32x4 *>(from.scal)[tid % (SCALAR_FLOATS / 4)];
    };
    auto load_dy = [&](int i, auto full) __attribute__((always_inline)) {
        dy.template load<full.value>(p.dy, b, (int64_t)i * C, 0, min(C, len - i * C), mine);
    };
    auto scalar = [&](int which, int at, int sub) __attribute__((always_inline)) {
        return *reinterpret_cast<const f32x4 *>(sc + which * C + 32 * at + 8 * quad + 4 * sub);
    };
    // As forward, the other way round: what is not finite goes into products as zeros, because later tokens have it too, times 0;
    // lost[] has the last token of a chunk from which a column has some, and everything up to it becomes a NaN (the chunks before it
    // start from a Z of NaNs).
    auto finite = [&](f32x4 (&x)[2]) __attribute__((always_inline)) {
        float f = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) f = fmaf(x[k >> 2][k & 3], 0.0f, f);
        if (__ballot(f != 0.0f) == 0) return;                       // (a NaN is not 0)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (!isfinite(x[k >> 2][k & 3])) {
                atomicMax(&lost[16 * tile + l16], 32 * half + 8 * quad + k);
                x[k >> 2][k & 3] = 0.0f;
            }
    };
    auto finite_dy = [&]() __attribute__((always_inline)) {          // (of the tokens that the own ones are summed over)
        float f = 0.0f;
#pragma unroll
        for (int k = 2 * half; k < 4; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) f = fmaf(dy.value(k, r), 0.0f, f);
        if (__ballot(f != 0.0f) == 0) return;
#pragma unroll
        for (int k = 2 * half; k < 4; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!isfinite(dy.value(k, r))) {
                    atomicMax(&lost[16 * tile + l16], 32 * (k >> 1) + 8 * quad + 4 * (k & 1) + r);
                    dy.v[k][r] = 0;
                }
    };
    auto lose = [&](f32x4 (&x)[2]) __attribute__((always_inline)) {
        const int upto = lost[16 * tile + l16];
        if (__ballot(upto >= 0) == 0) return;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (32 * half + 8 * quad + k <= upto) x[k >> 2][k & 3] = __builtin_nanf("");
    };
    // Z += (rows of keys)^T w over the tokens of half `f`
    auto into_state = [&](const Keys<NK, KF * 32> &t, int f, const bf16x8 (&w)[3]) __attribute__((always_inline)) {
        if (has)
#pragma unroll
            for (int o = 0; o < KO; ++o) {
                bf16x8 a[2][NK];
                t.cols(half + 2 * o, 0, f, a[0]);
                t.cols(half + 2 * o, 1, f, a[1]);
                multiply_rows<3>(Z[o], a, w);
                __builtin_amdgcn_sched_barrier(0);
            }
    };

    // Chunk i; `full`: whole, and so is chunk `then`, whose operands go out on the way
    auto step = [&](int i, int then, auto full) __attribute__((always_inline)) {
        const int64_t t0 = (int64_t)i * C, chunk = (b * p.n + i) * p.H + h;
        const int m = min(C, len - i * C);
        if constexpr (half == 1) {
            kr.template store<full.value, WIDE>(kt, m, p.Dk);
            qr.template store<full.value, WIDE>(qt, m, p.Dk);
            wr.store(wt);
            mr.store(mt);
            if (tid - NT < SCALAR_FLOATS / 4) reinterpret_cast<f32x4 *>(sc)[tid - NT] = sr;
        }
        __syncthreads();

        // K Z over the own rows: Y[0], [1] for the own tokens, [2], [3] for the other's
        const f32x4 out_k[2] = {scalar(OUT_K, half, 0), scalar(OUT_K, half, 1)}, beta[2] = {scalar(BETA, half, 0), scalar(BETA, half, 1)};
        f32x4 Y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) Y[k] = f32x4{0, 0, 0, 0};
        if (busy && has)
#pragma unroll
            for (int o = 0; o < KO; ++o) {
                bf16x8 z[3], a[4][NK];
#pragma unroll
                for (int k = 0; k < 4; ++k) kt.rows(half ^ (k >> 1), k & 1, half + 2 * o, a[k]);
                operand<3>(Z[o][0], Z[o][1], z);
                multiply_rows<3>(Y, a, z);
                __builtin_amdgcn_sched_barrier(0);
            }
        // exp(G_C) Z + Q^T (i dy); what Z was goes to memory
        auto fade = [&]() __attribute__((always_inline)) {
            const float whole = exp2_of(reinterpret_cast<const double *>(sc + SCALARS * C)[C - 1]);
#pragma unroll
            for (int o = 0; o < KO; ++o) {
                const int dk = 32 * (half + 2 * o);
                if (has) put_rows(Z[o], p.ds + (chunk * p.Dk + dk) * Dv + c, p.Dk - dk, Dv, in);
#pragma unroll
                for (int k = 0; k < 2; ++k) Z[o][k] *= whole;
            }
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                f32x4 d[2];
                bf16x8 w[3];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const f32x4 in_q = scalar(IN_Q, f, k);
#pragma unroll
                    for (int r = 0; r < 4; ++r) d[k][r] = in_q[r] * dy.value(2 * f + k, r);
                }
                operand<3>(d[0], d[1], w);
                into_state(qt, f, w);
            }
            if constexpr (full.value) load_dy(then, full);
        };
        bf16x8 y[2][NK];
        if (busy) {
            finite_dy();
#pragma unroll
            for (int f = 1 - half; f >= 0; --f) {       // (the second half's tokens, and for the first half its own)
                f32x4 d[2];
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int r = 0; r < 4; ++r) d[k][r] = dy.value(2 * (1 - f) + k, r);
                operand<NK>(d[0], d[1], y[1 - f]);
            }
        }
        if constexpr (L::shared) {
            if (busy) fade();
            __syncthreads();
        }
        if (busy) {
            to_other[0] = Y[2];
            to_other[64] = Y[3];
        }
        __syncthreads();

        // x = y - W^T (b y): the second half's tokens at once, the first's part of their own
        f32x4 X[2], U[2];
        bf16x8 u[3], w[3];
        auto outer = [&]() __attribute__((always_inline)) {
            const f32x4 in_k[2] = {scalar(IN_K, half, 0), scalar(IN_K, half, 1)};
#pragma unroll
            for (int k = 0; k < 2; ++k) U[k] = -in_k[k] * (beta[k] * X[k]);
            operand<3>(U[0], U[1], w);
        };
        auto results = [&]() __attribute__((always_inline)) {
            put_rows(X, p.dx + (chunk * C + 32 * half) * Dv + c, 32, Dv, in);
#pragma unroll
            for (int k = 0; k < 2; ++k) X[k] *= beta[k];
            put_column<full.value, T>(X, p.dv, b, t0, half, m, (int)min((int64_t)C, p.L - t0), h * Dv + c, in);
        };
        if (busy) {
            bf16x8 a[2][3];
            mt.cols(half, 0, 1, a[0]);
            mt.cols(half, 1, 1, a[1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) X[k] = (Y[k] + to_me[64 * k]) * out_k[k];
            multiply_rows<3>(X, a, y[1]);
            if constexpr (half == 0) {
                mt.cols(0, 0, 0, a[0]);
                mt.cols(0, 1, 0, a[1]);
                multiply_rows<3>(X, a, y[0]);
            }
            wt.cols(half, 0, half, a[0]);
            wt.cols(half, 1, half, a[1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) U[k] = beta[k] * X[k];
            finite(U);
            operand<3>(U[0], U[1], u);
            multiply_rows<3>(X, a, u);
            if constexpr (half == 1) {
                lose(X);
                outer();
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    one[64 * k] = u[k];
                    two[64 * k] = w[k];
                }
            } else if constexpr (!L::shared) {
                fade();
            }
        }
        __syncthreads();
        if constexpr (half == 1) {
            if constexpr (full.value) load(then, full);
            if (busy) {
                if constexpr (!L::shared) fade();
                into_state(kt, 1, w);
                results();
            }
        } else if (busy) {
            bf16x8 u1[3], a[2][3];
#pragma unroll
            for (int k = 0; k < 3; ++k) u1[k] = one[64 * k];
            wt.cols(0, 0, 1, a[0]);
            wt.cols(0, 1, 1, a[1]);
            multiply_rows<3>(X, a, u1);
            lose(X);
            outer();
#pragma unroll
            for (int k = 0; k < 3; ++k) one[64 * k] = w[k];
        }
        __syncthreads();
        if (busy) {
            if constexpr (half == 1) {
#pragma unroll
                for (int k = 0; k < 3; ++k) w[k] = one[64 * k];
                into_state(kt, 0, w);
            } else {
                bf16x8 w1[3];
#pragma unroll
                for (int k = 0; k < 3; ++k) w1[k] = two[64 * k];
                into_state(kt, 0, w);
                into_state(kt, 1, w1);
                results();
            }
            if (lost[16 * tile + l16] >= 0)
#pragma unroll
                for (int o = 0; o < KO; ++o)
#pragma unroll
                    for (int k = 0; k < 8; ++k) Z[o][k >> 2][k & 3] = __builtin_nanf("");
        }
        __syncthreads();
    };
    if (tid < 64) lost[tid] = -1;                           // (the first chunk's barrier is before the first use)
    const int whole_chunks = len / C;
    if (whole_chunks < n) {
        if constexpr (half == 1) load(n - 1, std::false_type());
        load_dy(n - 1, std::false_type());
        step(n - 1, n - 1, std::false_type());
    }
    if (whole_chunks > 0) {
        if constexpr (half == 1) load(whole_chunks - 1, std::true_type());
        load_dy(whole_chunks - 1, std::true_type());
        for (int i = whole_chunks - 1; i >= 0; --i) step(i, max(i - 1, 0), std::true_type());     // (the first one's again: no branch)
    }
    if (p.dh0 && has)
#pragma unroll
        for (int o = 0; o < KO; ++o) {
            const int dk = 32 * (half + 2 * o);
            put_rows(Z[o], p.dh0 + (head * p.Dk + dk) * Dv + c, p.Dk - dk, Dv, in);
        }
    const int cols = min(p.width, (int)Dv - c0);
    for (int64_t u = tid; u < (p.L - (int64_t)n * C) * cols; u += CHUNK_THREADS) {
        const int64_t t = (int64_t)n * C + u / cols;
        static_cast<T *>(p.dv.data)[b * p.dv.s0 + t * p.dv.s1 + h * Dv + c0 + u % cols] = (T)0.0f;
    }
}
template <typename T, int KF, bool WIDE>
__global__ __launch_bounds__(CHUNK_THREADS, 2) void merit_delta_back_chunks(DeltaParams p)
{
    extern __shared__ __attribute__((aligned(16))) __bf16 smem[];
    __shared__ int lost[64];
    if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 8) == 0) backward_half<T, KF, WIDE, 0>(p, smem, lost);
    else backward_half<T, KF, WIDE, 1>(p, smem, lost);
}

// ---------------------------------------------------------------------------
// chunks side by side: the gradients of q, k, g and beta; a workgroup a chunk of a head
// ---------------------------------------------------------------------------
// First the products along v's columns, 32 of them at a time: a wavefront takes 16 of the keys' columns of S_0 and Z straight from
// memory, LDS holds dy, x and u in terms.  Then those along the chunk's tokens, for which it holds K, Q and one matrix of 64 x 64
// after the other.  Results are kept times what a row goes through at the end: dQ scale / |q|, rows / |k|, cols / |k|, for which the
// matrices have the lengths of both of their tokens, and serve both ways round.  Through LDS they come into rows of eight values a
// thread, for the sums along the keys and the stores.
// 4096 chunks, 128 x 128, bfloat16: 424 us for 0.64 GB (1.5 TB/s).  A compute unit holds one workgroup of eight wavefronts, which pass
// its barriers together: LDS reads (each wavefront reads dy, x and u), vector instructions (about 120 us of them), products (76)
// and loads follow each other more than they overlap.  Asking for columns two turns ahead did not help, and spilled for 64 keys.
template <int KF> constexpr int grad_waves() { return KF < 4 ? 4 : 8; }
template <typename T, int KF, bool WIDE>
__global__ __launch_bounds__(64 * grad_waves<KF>(), 2) void merit_delta_grads(DeltaParams p)
{
    constexpr int NK = Terms<T>::n, RT = C / 16, WAVES = grad_waves<KF>(), THREADS = 64 * WAVES, OP = KF * 32 + 4;
    extern __shared__ __attribute__((aligned(16))) __bf16 smem[];
    __shared__ double G[C], sums[2][WAVES], suffix[C];
    __shared__ float invk[C], invq[C], beta[C];
    __shared__ int before[WAVES];
    typedef Tile<3, C, 32> TU;
    typedef Tile<NK, C, KF * 32> TK;
    const Tile<NK, C, 32> yt{smem};
    const TU xt{yt.at + Tile<NK, C, 32>::bytes / 2}, ut{xt.at + TU::bytes / 2};
    const TK kt{smem}, qt{kt.at + TK::bytes / 2};
    const Tile<3, C, C> wt{qt.at + TK::bytes / 2};
    float *const ot = reinterpret_cast<float *>(wt.at);        // [C][OP], in the place of the matrices

    const uint32_t id = blockIdx.x, h = id % (uint32_t)p.H, bi = id / (uint32_t)p.H;
    const uint32_t i = bi % (uint32_t)p.n;
    const int64_t b = bi / (uint32_t)p.n, t0 = (int64_t)i * C, Dv = p.Dv;
    const int kh = (int)h / p.each, m = min(C, tokens_of(p, b) - (int)t0), here = (int)min((int64_t)C, p.L - t0);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, quad = lane >> 4;
    // rows t of dq or dk, as they lie: the tensor's, or the value head's part in fp32
    auto put8 = [&](const Rows &out, int64_t which, int t, int c, const float (&v)[8]) __attribute__((always_inline)) {
        if (p.part) {
            float *to = p.part + ((which * p.B * p.L + b * p.L + t0 + t) * p.H + h) * p.Dk + c;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < p.Dk) to[e] = v[e];
            return;
        }
        T *to = static_cast<T *>(out.data) + b * out.s0 + (t0 + t) * out.s1 + (int64_t)kh * p.Dk + c;
        if (p.wide_out) {
            if (c >= p.Dk) return;
            typename Eight<T>::vec o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = (T)v[e];
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
                u32x4 w;
                __builtin_memcpy(&w, reinterpret_cast<const char *>(&o) + 16 * k, 16);
                reinterpret_cast<u32x4 *>(to)[k] = w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < p.Dk) to[e] = (T)v[e];
        }
    };
    if (m <= 0) {
        const float none[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (int u = tid; u < here * KF * 4; u += THREADS) {
            put8(p.dq, 0, u / (KF * 4), u % (KF * 4) * 8, none);
            put8(p.dk, 1, u / (KF * 4), u % (KF * 4) * 8, none);
        }
        if (tid < here) {
            if (p.dg.data) static_cast<float *>(p.dg.data)[b * p.dg.s0 + (t0 + tid) * p.dg.s1 + h] = 0.0f;
            static_cast<float *>(p.dbeta.data)[b * p.dbeta.s0 + (t0 + tid) * p.dbeta.s1 + h] = 0.0f;
        }
        return;
    }
    const float *scal = prepared(p, id).scal;
    if (tid < C) {
        G[tid] = reinterpret_cast<const double *>(scal + SCALARS * C)[tid];
        invk[tid] = scal[INV_K * C + tid];
        invq[tid] = scal[INV_Q * C + tid];
        beta[tid] = scal[BETA * C + tid];
    }
    const float *state = p.states + (int64_t)id * p.prep_stride + PREPARED_FLOATS, *kept = state + p.Dk * Dv;
    const float *zs = p.ds + (int64_t)id * p.Dk * Dv, *xs = p.dx + (int64_t)id * C * Dv;
    // a thread of the first four wavefronts moves eight values of a token of dy and x, of the last four (they may be the same) of u;
    // and every lane eight of the rows of S_0 and Z that are its own
    const bool first = tid < NT, second = tid >= THREADS - NT;
    const int tr = (tid & (NT - 1)) >> 2, tc = (tid & 3) * 8;
    const T *dyrow = static_cast<const T *>(p.dy.data) + b * p.dy.s0 + (t0 + min(tr, m - 1)) * p.dy.s1 + h * Dv;
    const float bt = scal[BETA * C + tr];
    const int row = 16 * wave + l16;
    const bool keys = wave < 2 * KF;                           // (the wavefront has a tile of keys)
    struct In {
        Eight<T> dy;
        Eight<float> x, d, s, z;
    };
    In in;
    auto load = [&](In &to, int c0) __attribute__((always_inline)) {
        const int left = (int)Dv - c0;
        to.dy = take8<WIDE, T>(dyrow + c0, tc, left);
        to.x = take8<WIDE, float>(xs + tr * Dv + c0, tc, left);
        to.d = take8<WIDE, float>(kept + tr * Dv + c0, tc, left);
        const int64_t at = (int64_t)min(row, p.Dk - 1) * Dv + c0;
        to.s = take8<WIDE, float>(state + at, 8 * quad, left);
        to.z = take8<WIDE, float>(zs + at, 8 * quad, left);
    };

    f32x4 dq[RT], rows[RT], cols[RT], dP[RT], dM[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) dP[rt] = dM[rt] = dq[rt] = rows[rt] = cols[rt] = f32x4{0, 0, 0, 0};
    // With eight wavefronts the first four have the rows of dP, the others those of dM
    const int own = wave & 3;
    const bool has_p = wave < 4, has_m = WAVES == 4 || wave >= 4;
    float db = 0.0f;
    double sz = 0.0;
    uint32_t held = 0;                                  // (bits of the state before the sequence's first chunk)
    const int end = ((int)Dv - 1) / 32 * 32;            // (the last turn's again behind it: no branch)
    auto turn = [&](In &now, int c0) __attribute__((always_inline)) {
        __syncthreads();
        bf16x8 st[3], zt[3];
        {
            const int left = (int)Dv - c0;
            const Eight<T> dy = keep8<WIDE, T>(now.dy, tc, tr < m ? left : 0);
            const Eight<float> x = keep8<WIDE, float>(now.x, tc, left), s = keep8<WIDE, float>(now.s, 8 * quad, row < p.Dk ? left : 0),
                               z = keep8<WIDE, float>(now.z, 8 * quad, row < p.Dk ? left : 0);
            Eight<float> d = keep8<WIDE, float>(now.d, tc, left);
            bf16x8 o[NK], o3[3];
            if (first) {
                terms8<T>(dy, o);
                yt.put8(tr, tc, o);
                terms8<float>(x, o3);
                xt.put8(tr, tc, o3);
            }
            if (second) {
#pragma unroll
                for (int e = 0; e < 8; ++e) db = fmaf(x.v[e], d.v[e], db);
                d.v *= bt;
                terms8<float>(d, o3);
                ut.put8(tr, tc, o3);
            }
            float f = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) f = fmaf(s.v[e], z.v[e], f);
            sz += (double)f;
            if (i == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e) held |= __builtin_bit_cast(uint32_t, s.v[e]) << 1;
            terms8<float>(s, st);
            terms8<float>(z, zt);
        }
        load(now, min(c0 + 32, end));
        __syncthreads();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            bf16x8 a[NK], a3[3], u[3];
            yt.rows(16 * rt, 0, a);
            xt.rows(16 * rt, 0, a3);
            ut.rows(16 * rt, 0, u);
            if (keys) {
                multiply<3>(dq[rt], a, st);
                multiply<3>(rows[rt], a3, st);
                multiply<3>(cols[rt], u, zt);
            }
            if (rt <= own) {
                if (has_p) {
                    yt.rows(16 * own, 0, a);
                    multiply<3>(dP[rt], a, u);
                }
                if (has_m) {
                    xt.rows(16 * own, 0, a3);
                    multiply<3>(dM[rt], a3, u);
                }
            }
        }
    };
    load(in, 0);
    for (int c0 = 0; c0 <= end; c0 += 32) turn(in, c0);
    // K and Q: a unit of eight values a thread and turn
    constexpr int key_units = C * KF * 4 / THREADS;
    static_assert(key_units >= 1, "");
    Eight<T> ke[key_units], qe[key_units];
#pragma unroll
    for (int n = 0; n < key_units; ++n) {
        const int u = tid + n * THREADS, r = u / (KF * 4), c = u % (KF * 4) * 8, D = p.Dk;
        const T *krow = static_cast<const T *>(p.k.data) + b * p.k.s0 + (t0 + min(r, m - 1)) * p.k.s1 + (int64_t)kh * D;
        const T *qrow = static_cast<const T *>(p.q.data) + b * p.q.s0 + (t0 + min(r, m - 1)) * p.q.s1 + (int64_t)kh * D;
        if (p.wide_qk) {
            ke[n] = take8<true, T>(krow, c, D);
            qe[n] = take8<true, T>(qrow, c, D);
        } else {
            ke[n] = take8<false, T>(krow, c, D);
            qe[n] = take8<false, T>(qrow, c, D);
        }
    }
    db += lane_xor<0>(db);
    db += lane_xor<1>(db);
    if (!keys) sz = 0.0;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) sz += __shfl_xor(sz, k);
    if (lane == 0) sums[0][wave] = sz;
    const bool any = __ballot(held != 0) != 0;
    if (lane == 0) before[wave] = i > 0 || any;
    __syncthreads();            // (the first part's LDS is free)
#pragma unroll
    for (int n = 0; n < key_units; ++n) {
        const int u = tid + n * THREADS, r = u / (KF * 4), c = u % (KF * 4) * 8, there = r < m ? p.Dk : 0;
        bf16x8 o[NK];
        terms8<T>(p.wide_qk ? keep8<true, T>(ke[n], c, there) : keep8<false, T>(ke[n], c, there), o);
        kt.put8(r, c, o);
        terms8<T>(p.wide_qk ? keep8<true, T>(qe[n], c, there) : keep8<false, T>(qe[n], c, there), o);
        qt.put8(r, c, o);
    }
    // the matrices' rows of the wavefront
    {
        float tk[4], tq[4], tb[4];
        double gt[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = 16 * own + 4 * quad + r;
            tk[r] = invk[t];
            tq[r] = invq[t] * p.scale;
            tb[r] = -beta[t] * tk[r];
            gt[r] = G[t];
        }
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            if (j > (own | 1)) continue;
            const int c = 16 * j + l16;
            const float ck = invk[c];
            const double gc = G[c];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 16 * own + 4 * quad + r;
                const float f = c <= t ? exp2_of(gt[r] - gc) * ck : 0.0f;
                dP[j][r] = c <= t ? f * tq[r] * dP[j][r] : 0.0f;
                dM[j][r] = c < t ? f * tb[r] * dM[j][r] : 0.0f;
                if (has_p) wt.put1(t, c, dP[j][r]);
            }
        }
    }
    // rows' factors
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const f32x4 in_q = *reinterpret_cast<const f32x4 *>(scal + IN_Q * C + 16 * rt + 4 * quad);
        const f32x4 in_k = *reinterpret_cast<const f32x4 *>(scal + IN_K * C + 16 * rt + 4 * quad);
        const f32x4 out_k = *reinterpret_cast<const f32x4 *>(scal + OUT_K * C + 16 * rt + 4 * quad);
        const f32x4 bb = *reinterpret_cast<const f32x4 *>(scal + BETA * C + 16 * rt + 4 * quad);
        dq[rt] *= in_q;
        rows[rt] *= -in_k * bb;
        cols[rt] *= out_k;
    }
    __syncthreads();
    // K.(o u Z^T), for the last token's G
    double kz = 0.0;
    if (keys) {
        float f = 0.0f;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) f = fmaf(kt.value(16 * rt + 4 * quad + r, row), cols[rt][r], f);
        kz = (double)f;
    }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) kz += __shfl_xor(kz, k);
    if (lane == 0) sums[1][wave] = kz;

    // to += W B (rows at or before the diagonal), and += W^T B
    auto along = [&](f32x4 (&to)[RT], const bf16x8 (&o)[2][NK]) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int rt = 2 * f; rt < RT; ++rt) {
                bf16x8 a[3];
                wt.rows(16 * rt, 32 * f, a);
                multiply<3>(to[rt], a, o[f]);
            }
    };
    auto across = [&](f32x4 (&to)[RT], const bf16x8 (&o)[2][NK]) __attribute__((always_inline)) {
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
            for (int rt = 0; rt < 2 * f + 2; ++rt) {
                bf16x8 a[3];
                wt.cols(32 * f, 16 * rt, a);
                multiply<3>(to[rt], a, o[f]);
            }
    };
    bf16x8 ko[2][NK];
    if (keys) {
        bf16x8 qo[2][NK];
#pragma unroll
        for (int f = 0; f < 2; ++f) {
            kt.cols(32 * f, 16 * wave, ko[f]);
            qt.cols(32 * f, 16 * wave, qo[f]);
        }
        along(dq, ko);
        across(cols, qo);
    }
    __syncthreads();
    if (has_m)
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            if (j > (own | 1)) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) wt.put1(16 * own + 4 * quad + r, 16 * j + l16, dM[j][r]);
        }
    __syncthreads();
    if (keys) {
        along(rows, ko);
        across(cols, ko);
    }
    // Eight values of a token's row a thread and turn, for the sums along the keys (its KF * 4 lanes have the row) and the stores
    constexpr int units = C * KF * 4 / THREADS;
    auto by_rows = [&](const f32x4 (&v)[RT], float (&o)[units][8]) __attribute__((always_inline)) {
        __syncthreads();
        if (keys)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int r = 0; r < 4; ++r) ot[(16 * rt + 4 * quad + r) * OP + row] = v[rt][r];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < units; ++n) {
            const int u = tid + n * THREADS;
            const f32x4 *from = reinterpret_cast<const f32x4 *>(ot + u / (KF * 4) * OP + u % (KF * 4) * 8);
            const f32x4 lo = from[0], hi = from[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[n][e] = lo[e];
                o[n][4 + e] = hi[e];
            }
        }
    };
    auto values = [&](const TK &t, int r, int c, float (&o)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll
        for (int k = NK - 1; k >= 0; --k) {
            const bf16x8 w = *reinterpret_cast<const bf16x8 *>(t.at + k * TK::plane + r * TK::pitch + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += (float)w[e];
        }
    };
    auto dot = [&](const float (&a)[8], const float (&b)[8]) __attribute__((always_inline)) {
        float v = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) v = fmaf(a[e], b[e], v);
        return sum_lanes(v, KF * 4);
    };
    float vq[units][8], va[units][8], vc[units][8];
    by_rows(dq, vq);
    by_rows(rows, va);
    by_rows(cols, vc);
#pragma unroll
    for (int n = 0; n < units; ++n) {
        const int u = tid + n * THREADS, t = u / (KF * 4), c = u % (KF * 4) * 8;
        float qv[8], kv[8];
        values(qt, t, c, qv);
        values(kt, t, c, kv);
        const float dotq = dot(qv, vq[n]), dota = dot(kv, va[n]), dotc = dot(kv, vc[n]);
        if (c == 0) suffix[t] = (double)dotq + (double)dota - (double)dotc;
        // through the lengths
        const float fq = p.unit ? invq[t] * invq[t] * dotq : 0.0f, fk = p.unit ? invk[t] * invk[t] * (dota + dotc) : 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            vq[n][e] = t < m ? fmaf(-fq, qv[e], vq[n][e]) : 0.0f;
            va[n][e] = t < m ? fmaf(-fk, kv[e], va[n][e] + vc[n][e]) : 0.0f;
        }
        if (t < here) {
            put8(p.dq, 0, t, c, vq[n]);
            put8(p.dk, 1, t, c, va[n]);
        }
    }
    __syncthreads();
    if (wave == 0) {
        double a = suffix[lane];
        if (lane == C - 1) {
            double f = 0.0, g = 0.0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                f += sums[0][w];
                g += sums[1][w];
            }
            a += (double)exp2_of(G[C - 1]) * f + g;
        }
#pragma unroll
        for (int k = 1; k < C; k *= 2) {
            const double o = __shfl_down(a, k);
            if (lane + k < C) a += o;
        }
        // Before the first token of a state of zeros there is nothing to fade: no gradient, where the sums cancel to their roundings
        int some = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) some |= before[w];
        if (lane == 0 && !some && isfinite(a)) a = 0.0;
        if (lane < here && p.dg.data)
            static_cast<float *>(p.dg.data)[b * p.dg.s0 + (t0 + lane) * p.dg.s1 + h] = lane < m ? (float)a : 0.0f;
    }
    if (second && (tid & 3) == 0 && tr < here)
        static_cast<float *>(p.dbeta.data)[b * p.dbeta.s0 + (t0 + tr) * p.dbeta.s1 + h] = tr < m ? db : 0.0f;
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
    constexpr int lds = BackwardLds<T, KF>::bytes;
    static_assert(lds + 256 <= 160 * 1024, "");
    p.width = delta_width(p.B * p.H, p.Dv, 0);
    p.slices = delta_slices(p.width, p.Dv, 0);
    const unsigned grid = (unsigned)(p.B * p.H * p.slices);
    if (p.wide_qk) merit_delta_back_chunks<T, KF, true><<<grid, CHUNK_THREADS, lds, s>>>(p);
    else merit_delta_back_chunks<T, KF, false><<<grid, CHUNK_THREADS, lds, s>>>(p);
    return hipGetLastError();
}
template <typename T, int KF> hipError_t grads_of(const DeltaParams &p, hipStream_t s)
{
    constexpr int NK = Terms<T>::n;
    constexpr int one = Tile<NK, C, 32>::bytes + 2 * Tile<3, C, 32>::bytes;
    constexpr int matrix = Tile<3, C, C>::bytes, out = C * (KF * 32 + 4) * 4;
    constexpr int two = 2 * Tile<NK, C, KF * 32>::bytes + (matrix > out ? matrix : out);
    constexpr int lds = one > two ? one : two;
    static_assert(lds + 3 * 1024 <= 160 * 1024, "");
    const unsigned grid = (unsigned)(p.B * p.n * p.H);
    if (p.wide_v) merit_delta_grads<T, KF, true><<<grid, 64 * grad_waves<KF>(), lds, s>>>(p);
    else merit_delta_grads<T, KF, false><<<grid, 64 * grad_waves<KF>(), lds, s>>>(p);
    return hipGetLastError();
}
template <typename T, int KF> hipError_t backward_of(const DeltaParams &p, hipStream_t s)
{
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
