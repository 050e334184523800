// The gated delta rule, forward: what a chunk's tokens do to each other (merit_delta_prepare), chunk after chunk
// (merit_delta_chunks), one token (merit_delta_token).  The formulas stand in delta.h.
#pragma once

#include "delta.h"

namespace merit {
namespace delta {

// ---------------------------------------------------------------------------
// chunks side by side: a workgroup a chunk of a head
// ---------------------------------------------------------------------------
// It leaves -W and P in terms, and the tokens' factors.  W is found in blocks of 16 x 16 on v_mfma_f32_16x16x4_f32: those on the
// diagonal by forward substitution, a thread a column, the rest from them.  Keys of 128, bfloat16, 4096 chunks: 73 us, 0.24 GB (3.3
// TB/s); vector instructions are busy more than half of that time, and what waits are the steps for each other.
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
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, quad = lane >> 4;
    const Prepared to = prepared(p, id);
    float *const scal = to.scal;

    // Two rows' loads in a wavefront: keys to LDS, their squares' sums over the lanes of a row
    ChunkRows<T, KF, NT> kr;
    kr.template load<false, WIDE>(p.k, b, t0, m, kh, p.Dk);
    const int own = 16 * wave + l16;
    const T *qrow = static_cast<const T *>(p.q.data) + b * p.q.s0 + (t0 + min(own, m - 1)) * p.q.s1 + (int64_t)kh * p.Dk;
    Eight<T> qe[KF];
#pragma unroll
    for (int f = 0; f < KF; ++f) qe[f] = take8<WIDE, T>(qrow, 32 * f + 8 * quad, p.Dk);
    if (wave == 0) {
        double g = 0.0;
        float bt = 0.0f;
        if (lane < m) {
            if (p.g.data) g = log2_decay(static_cast<const float *>(p.g.data)[b * p.g.s0 + (t0 + lane) * p.g.s1 + h]);
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
#pragma unroll
    for (int f = 0; f < KF; ++f) qe[f] = keep8<WIDE, T>(qe[f], 32 * f + 8 * quad, own < m ? p.Dk : 0);
    if (p.unit) {
#pragma unroll
        for (int u = 0; u < ChunkRows<T, KF, NT>::units; ++u) {
            const Eight<T> x = kr.template value<false, WIDE>(u, m, p.Dk);
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fmaf((float)x.v[e], (float)x.v[e], s);
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
    kr.template store<false, WIDE>(kt, m, p.Dk);
    __syncthreads();

    if (tid < C) {
        const double g = G[tid], last = G[C - 1];
        const float in = exp2_of(g);
        scal[IN_K * C + tid] = in * invk[tid];
        scal[BETA * C + tid] = beta[tid];
        scal[OUT_K * C + tid] = exp2_of(last - g) * invk[tid];
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
            const float f = j <= t ? exp2_of(gt - G[j]) * lens[r] : 0.0f;
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
                *reinterpret_cast<bf16x4 *>(to.mix + k * TRIANGLE + triangle_at(t, j0)) = out[k];
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
        for (int k = 0; k < 2; ++k) {
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = lost ? __builtin_nanf("") : below ? -x[r][c0 + 8 * k + j] : 0.0f;
            bf16x8 o[3];
            split8<3>(e, o);
#pragma unroll
            for (int n = 0; n < 3; ++n) *reinterpret_cast<bf16x8 *>(to.w + n * TRIANGLE + triangle_at(r, c0 + 8 * k)) = o[n];
        }
    }
}

// ---------------------------------------------------------------------------
// one chunk after the other: two wavefronts 16 columns of a head's state
// ---------------------------------------------------------------------------
// The columns of a state do not depend on each other.  Two wavefronts of a SIMD have 16 of them: each one half of a chunk's
// tokens and every other 32 rows of the state, in registers, so that one issues while the other waits (a wavefront alone issues
// an instruction in four cycles, 1.4 thousand a chunk; one for all tokens took 1.25 times as long).  They meet for the sums over
// the state's rows, for what the first half's tokens leave for the second's, and for what both leave for the state.  LDS holds
// the other operands, K, Q and the two triangular matrices, for the eight wavefronts of a workgroup; the next chunk's are on
// their way in registers meanwhile. Bound by the chain of a chunk's products and barriers, bfloat16, states of 128 x 128: 4.3 us
// a chunk with one pair at work (16 heads of 8191 tokens 551 us), 8.6 with four in every compute unit, LDS, vector and matrix
// instructions a quarter of the time each (128 heads of 2048 with the states kept 274 us, 0.79 GB, 2.9 TB/s; without 188).  Few long
// sequences go in segments side by side (16 heads of 8191: 108 us for what eight segments do to a state, 22 to join them, 92 from their
// first states on).  P and u go into y with three terms as everything else does: two, enough for the rounding of a 16-bit y itself,
// lost 2^-17 of each of a sum's terms, which shows where they cancel (128 heads of 2048, no states kept, 246 against 259 us a call).
constexpr int CHUNK_THREADS = 512;
template <typename T, int KF> struct ForwardLds {
    static constexpr int NK = Terms<T>::n;
    static constexpr int k = 0, w = k + Keys<NK, KF * 32>::bytes, mix = w + Triangle<3>::bytes, scal = mix + Triangle<3>::bytes,
                         q = scal + SCALAR_FLOATS * 4, past_q = q + Keys<NK, KF * 32>::bytes;
    // what the wavefronts of a pair hand each other: 4 KB to each, w and u of the first; where LDS is full, in the place of Q
    static constexpr int pair = (8 + 3 + 3) * 1024;
    static constexpr bool shared = past_q + 4 * pair + 256 > 160 * 1024;
    static constexpr int hand = shared ? q : past_q;
    static constexpr int bytes = hand + 4 * pair > past_q ? hand + 4 * pair : past_q;
};
// Where a segment's first state is, and the transition of one that is neither the first nor the last
__device__ __forceinline__ float *segment_state(const DeltaParams &p, int seg) { return p.seg_state + seg * p.B * p.H * p.Dk * p.Dv; }
__device__ __forceinline__ float *segment_through(const DeltaParams &p, int seg)
{
    return p.seg_state + delta_segment_floats(p, p.segments, seg - 1);
}
// What a launch leaves: y and the last state; the same, and what the backward pass takes; what a segment does to a state
enum Leaves { RESULTS, KEPT, SEGMENT };
// (a half at a time is compiled: every place in LDS is then a lane's base and a constant)
template <typename T, int KF, bool WIDE, Leaves LEAVES, int half>
__device__ __forceinline__ void forward_half(const DeltaParams &p, __bf16 *smem, int *lost)
{
    typedef ForwardLds<T, KF> L;
    constexpr int NK = L::NK, KO = KF < 2 ? 1 : KF / 2;
    constexpr bool KEEP = LEAVES == KEPT, PASS = LEAVES == SEGMENT;
    char *const lds = reinterpret_cast<char *>(smem);
    const Keys<NK, KF * 32> kt{reinterpret_cast<__bf16 *>(lds + L::k)}, qt{reinterpret_cast<__bf16 *>(lds + L::q)};
    const Triangle<3> wt{reinterpret_cast<__bf16 *>(lds + L::w)}, mt{reinterpret_cast<__bf16 *>(lds + L::mix)};
    float *const sc = reinterpret_cast<float *>(lds + L::scal);

    const uint32_t id = blockIdx.x, h = id / (uint32_t)p.slices % (uint32_t)p.H;
    const int64_t b = id / (uint32_t)p.slices / (uint32_t)p.H;
    const int kh = (int)h / p.each, len = tokens_of(p, b), n = (len + C - 1) / C;
    // (a wavefront's number is said to be the same for its lanes: branches on it skip, and leave the lanes' mask as it is.  Behind one
    // that masks lanes, the compiler put a copy of a register in front of the mask's restoring, and wavefronts that skip kept an
    // old value: in fp32 with rows off 16 bytes and states kept, rows moved by wavefronts without columns were wrong.)
    const int tid = threadIdx.x, lane = tid & 63, tile = __builtin_amdgcn_readfirstlane(tid >> 6 & 3), l16 = lane & 15, quad = lane >> 4;
    const int64_t head = b * p.H + h, Dv = p.Dv;
    // a segment of the sequence's chunks; its transition, what comes of the unit matrix where v is zeros, has slices behind those of v
    const int seg = (int)blockIdx.y, i0 = seg * p.seg_chunks, i1 = min(n, i0 + p.seg_chunks), last = n > 0 ? (n - 1) / p.seg_chunks : 0;
    const int slice = (int)(id % (uint32_t)p.slices), of_v = (p.Dv + p.width - 1) / p.width;
    const bool through = PASS && slice >= of_v;
    const int64_t cols = through ? p.Dk : Dv;
    const int c0 = (slice - (through ? of_v : 0)) * p.width, c = c0 + 16 * tile + l16;
    const bool busy = 16 * tile < p.width && c0 + 16 * tile < cols, in = busy && c < cols, has = half < KF;
    if (PASS ? through && (seg == 0 || seg >= last) : seg > last) return;
    f32x4 *const to_me = reinterpret_cast<f32x4 *>(lds + L::hand + tile * L::pair + half * 4096) + lane;
    f32x4 *const to_other = reinterpret_cast<f32x4 *>(lds + L::hand + tile * L::pair + (1 - half) * 4096) + lane;
    bf16x8 *const first = reinterpret_cast<bf16x8 *>(lds + L::hand + tile * L::pair) + lane;                  // b x of the first
    bf16x8 *const second = reinterpret_cast<bf16x8 *>(lds + L::hand + tile * L::pair + 4096) + lane;          // w of the second
    bf16x8 *const third = reinterpret_cast<bf16x8 *>(lds + L::hand + tile * L::pair + 8192) + lane;           // w and u of the first

    f32x4 S[KO][2];
#pragma unroll
    for (int o = 0; o < KO; ++o) {
        const int dk = 32 * (half + 2 * o);
        // (later segments start from what merit_delta_join left, and the first from a copy: h_last may be h0)
        const float *from = p.h0;
        if (PASS && seg > 0) from = nullptr;
        if (!PASS && (seg > 0 || (p.segments > 1 && p.h0))) from = segment_state(p, seg);
        get_rows(S[o], from ? from + (head * p.Dk + dk) * Dv + c : nullptr, p.Dk - dk, Dv, in && !through);
        if (PASS && seg == 0 && p.h0 && has)
            put_rows(S[o], segment_state(p, 0) + (head * p.Dk + dk) * Dv + c, p.Dk - dk, Dv, in);
        if (through)
#pragma unroll
            for (int k = 0; k < 8; ++k) S[o][k >> 2][k & 3] = dk + 8 * quad + k == c ? 1.0f : 0.0f;
    }
    if (PASS && seg >= last) return;
    const int64_t mine = h * Dv + min((int64_t)c, Dv - 1);         // (a lane without a column: any that is there)
    // (the first half's wavefronts, which wait for the others later, move what the next chunk needs)
    ChunkRows<T, KF, NT> kr, qr;
    TriangleRows<3, NT> wr, mr;
    f32x4 sr;
    ChunkColumn<T, 1> v;
    auto load = [&](int i, auto full) __attribute__((always_inline)) {
        const int m = min(C, len - i * C);
        kr.template load<full.value, WIDE>(p.k, b, (int64_t)i * C, m, kh, p.Dk);
        if (!PASS) qr.template load<full.value, WIDE>(p.q, b, (int64_t)i * C, m, kh, p.Dk);
        const Prepared from = prepared(p, (b * p.n + i) * p.H + h);
        wr.load(from.w);
        if (!PASS) mr.load(from.mix);
        sr = reinterpret_cast<const f32x4 *>(from.scal)[tid % (SCALAR_FLOATS / 4)];
    };
    auto load_v = [&](int i, auto full) __attribute__((always_inline)) {
        v.template load<full.value>(p.v, b, (int64_t)i * C, half, min(C, len - i * C), mine);
    };
    auto scalar = [&](int which, int sub) __attribute__((always_inline)) {
        return *reinterpret_cast<const f32x4 *>(sc + which * C + 32 * half + 8 * quad + 4 * sub);
    };
    // Values that are not finite go into products as zeros, because those of earlier tokens have them too, times 0; lost[] has the
    // first token of a chunk from which a column has some, and everything from there on becomes a NaN (the chunks behind it start
    // from a state of NaNs).
    auto finite = [&](f32x4 (&x)[2]) __attribute__((always_inline)) {
        float f = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) f = fmaf(x[k >> 2][k & 3], 0.0f, f);
        if (__ballot(f != 0.0f) == 0) return;                       // (a NaN is not 0)
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (!isfinite(x[k >> 2][k & 3])) {
                atomicMin(&lost[16 * tile + l16], 32 * half + 8 * quad + k);
                x[k >> 2][k & 3] = 0.0f;
            }
    };
    auto lose = [&](f32x4 (&x)[2], int from) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (32 * half + 8 * quad + k >= from) x[k >> 2][k & 3] = __builtin_nanf("");
    };
    // S += K^T w over the tokens of half `f`
    auto into_state = [&](int f, const bf16x8 (&w)[3]) __attribute__((always_inline)) {
        if (has)
#pragma unroll
            for (int o = 0; o < KO; ++o) {
                bf16x8 a[2][NK];
                kt.cols(half + 2 * o, 0, f, a[0]);
                kt.cols(half + 2 * o, 1, f, a[1]);
                multiply_rows<3>(S[o], a, w);
                __builtin_amdgcn_sched_barrier(0);
            }
    };

    // Chunk i; `full`: whole, and so is chunk `then`, whose operands go out on the way
    auto step = [&](int i, int then, auto full) __attribute__((always_inline)) {
        const int64_t t0 = (int64_t)i * C, chunk = (b * p.n + i) * p.H + h;
        const int m = min(C, len - i * C);
        if constexpr (half == 0) {
            kr.template store<full.value, WIDE>(kt, m, p.Dk);
            wr.store(wt);
            if (!PASS) {
                qr.template store<full.value, WIDE>(qt, m, p.Dk);
                mr.store(mt);
            }
            if (tid < SCALAR_FLOATS / 4) reinterpret_cast<f32x4 *>(sc)[tid] = sr;
        }
        __syncthreads();

        // K S and Q S over the own rows of the state: X, Y[0], [1] for the own tokens, [2], [3] for the other's
        const f32x4 in_k[2] = {scalar(IN_K, 0), scalar(IN_K, 1)}, beta[2] = {scalar(BETA, 0), scalar(BETA, 1)};
        f32x4 X[4], Y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) X[k] = Y[k] = f32x4{0, 0, 0, 0};
        if (busy && has)
#pragma unroll
            for (int o = 0; o < KO; ++o) {
                bf16x8 s[3], a[4][NK];
#pragma unroll
                for (int k = 0; k < 4; ++k) kt.rows(half ^ (k >> 1), k & 1, half + 2 * o, a[k]);
                operand<3>(S[o][0], S[o][1], s);
                multiply_rows<3>(X, a, s);
                __builtin_amdgcn_sched_barrier(0);
                if (PASS) continue;
#pragma unroll
                for (int k = 0; k < 4; ++k) qt.rows(half ^ (k >> 1), k & 1, half + 2 * o, a[k]);
                multiply_rows<3>(Y, a, s);
                __builtin_amdgcn_sched_barrier(0);
            }
        if constexpr (L::shared) __syncthreads();
        if (busy) {
            to_other[0] = X[2];
            to_other[64] = X[3];
            if (!PASS) {
                to_other[128] = Y[2];
                to_other[192] = Y[3];
            }
        }
        __syncthreads();

        // d = r - W (b r), u, w = what goes into the state: the first half's tokens at once, the second's part of their own
        f32x4 D[2], U[2], O[2];
        bf16x8 x[3], w[3], u[3];
        if (busy) {
            bf16x8 a[2][3];
            wt.rows(half, 0, half, a[0]);
            wt.rows(half, 1, half, a[1]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x4 sum = X[k] + to_me[64 * k];
#pragma unroll
                for (int r = 0; r < 4; ++r) D[k][r] = fmaf(-in_k[k][r], sum[r], through ? 0.0f : v.value(k, r));
                O[k] = beta[k] * D[k];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (!PASS) Y[k] += to_me[128 + 64 * k];
            if constexpr (full.value) load_v(then, full);
            finite(O);
            operand<3>(O[0], O[1], x);
            multiply_rows<3>(D, a, x);
        }
        auto outer = [&]() __attribute__((always_inline)) {
            const f32x4 out_k[2] = {scalar(OUT_K, 0), scalar(OUT_K, 1)};
#pragma unroll
            for (int k = 0; k < 2; ++k) U[k] = beta[k] * D[k];
            finite(U);
#pragma unroll
            for (int k = 0; k < 2; ++k) O[k] = out_k[k] * U[k];
            operand<3>(O[0], O[1], w);
            if (!PASS) operand<3>(U[0], U[1], u);
        };
        if (busy && half == 0) {
            const int from = lost[16 * tile + l16];
            if (__ballot(from < C) != 0) lose(D, from);
            outer();
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                first[64 * k] = x[k];
                third[64 * k] = w[k];
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (!PASS) third[192 + 64 * k] = u[k];
        }
        __syncthreads();
        // the state before the chunk is not needed any more, but by those who keep it
        auto fade = [&]() __attribute__((always_inline)) {
            if (KEEP && has)
#pragma unroll
                for (int o = 0; o < KO; ++o) {
                    const int dk = 32 * (half + 2 * o);
                    put_rows(S[o], p.states + chunk * p.prep_stride + PREPARED_FLOATS + dk * Dv + c, p.Dk - dk, Dv, in);
                }
            const float whole = exp2_of(reinterpret_cast<const double *>(sc + SCALARS * C)[C - 1]);
#pragma unroll
            for (int o = 0; o < KO; ++o)
#pragma unroll
                for (int k = 0; k < 2; ++k) S[o][k] *= whole;
        };
        auto results = [&]() __attribute__((always_inline)) {
            bf16x8 a[2][3];
            mt.rows(half, 0, half, a[0]);
            mt.rows(half, 1, half, a[1]);
            f32x4 y[2] = {Y[0], Y[1]};
            multiply_rows<3>(y, a, u);
            const int from = lost[16 * tile + l16];
            if (__ballot(from < C) != 0) lose(y, from);
            put_column<full.value, T>(y, p.y, b, t0, half, m, (int)min((int64_t)C, p.L - t0), h * Dv + c, in);
            if (KEEP) put_rows(D, p.states + chunk * p.prep_stride + PREPARED_FLOATS + (p.Dk + 32 * half) * Dv + c, 32, Dv, in);
        };
        if constexpr (half == 0) {
            if constexpr (full.value) load(then, full);
            if (busy) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (!PASS) Y[k] *= scalar(IN_Q, k);
                fade();
                into_state(0, w);
                if (!PASS) results();
            }
        } else if (busy) {
            bf16x8 x0[3], a[2][3];
#pragma unroll
            for (int k = 0; k < 3; ++k) x0[k] = first[64 * k];
            wt.rows(1, 0, 0, a[0]);
            wt.rows(1, 1, 0, a[1]);
            const int from = lost[16 * tile + l16];
            multiply_rows<3>(D, a, x0);
            if (__ballot(from < C) != 0) lose(D, from);
            outer();
#pragma unroll
            for (int k = 0; k < 3; ++k) second[64 * k] = w[k];
        }
        __syncthreads();
        if (busy) {
            if constexpr (half == 0) {
#pragma unroll
                for (int k = 0; k < 3; ++k) w[k] = second[64 * k];
                into_state(1, w);
            } else {
                bf16x8 w0[3], u0[3], a[2][3];
#pragma unroll
                for (int k = 0; k < 3; ++k) w0[k] = third[64 * k];
                fade();
                into_state(1, w);
                into_state(0, w0);
                if constexpr (!PASS) {
#pragma unroll
                    for (int k = 0; k < 3; ++k) u0[k] = third[192 + 64 * k];
                    mt.rows(1, 0, 0, a[0]);
                    mt.rows(1, 1, 0, a[1]);
                    f32x4 y[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) y[k] = Y[k] * scalar(IN_Q, k);
                    multiply_rows<3>(y, a, u0);
                    Y[0] = y[0];
                    Y[1] = y[1];
                    results();
                }
            }
            if (lost[16 * tile + l16] < C)
#pragma unroll
                for (int o = 0; o < KO; ++o)
#pragma unroll
                    for (int k = 0; k < 8; ++k) S[o][k >> 2][k & 3] = __builtin_nanf("");
        }
        __syncthreads();
    };
    if (tid < 64) lost[tid] = C;
    const int whole = min(len / C, i1);                     // (the chunks from there on: at most one, the sequence's last)
    if (whole > i0) {
        if constexpr (half == 0) load(i0, std::true_type());
        load_v(i0, std::true_type());
        for (int i = i0; i < whole; ++i) step(i, min(i + 1, whole - 1), std::true_type());      // (the last one's again: no branch)
    }
    if constexpr (PASS) {
        const int64_t line = through ? delta_pitch(p) : Dv;
        float *const to = through ? segment_through(p, seg) + head * p.Dk * delta_pitch(p) : segment_state(p, seg + 1) + head * p.Dk * Dv;
        if (has)
#pragma unroll
            for (int o = 0; o < KO; ++o) {
                const int dk = 32 * (half + 2 * o);
                put_rows(S[o], to + dk * line + c, p.Dk - dk, line, in);
            }
        return;
    }
    if (whole < i1) {
        if constexpr (half == 0) load(n - 1, std::false_type());
        load_v(n - 1, std::false_type());
        step(n - 1, n - 1, std::false_type());
    }
    if (seg < last) return;
    if (p.h_last && has)
#pragma unroll
        for (int o = 0; o < KO; ++o) {
            const int dk = 32 * (half + 2 * o);
            put_rows(S[o], p.h_last + (head * p.Dk + dk) * Dv + c, p.Dk - dk, Dv, in);
        }
    // zeros behind the sequence's last chunk
    const int wide = min(p.width, (int)Dv - c0);
    for (int64_t u = tid; u < (p.L - (int64_t)n * C) * wide; u += CHUNK_THREADS) {
        const int64_t t = (int64_t)n * C + u / wide;
        static_cast<T *>(p.y.data)[b * p.y.s0 + t * p.y.s1 + h * Dv + c0 + u % wide] = (T)0.0f;
    }
}
template <typename T, int KF, bool WIDE, Leaves LEAVES>
__global__ __launch_bounds__(CHUNK_THREADS, 2) void merit_delta_chunks(DeltaParams p)
{
    extern __shared__ __attribute__((aligned(16))) __bf16 smem[];
    __shared__ int lost[64];
    if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 8) == 0) forward_half<T, KF, WIDE, LEAVES, 0>(p, smem, lost);
    else forward_half<T, KF, WIDE, LEAVES, 1>(p, smem, lost);
}

// The states that segments start from, one after the other: S <- A S + E, with the segment's transition A and what it makes of a state
// of zeros, E, in whose place the result goes.  A workgroup 16 columns of a head, a wavefront 16 rows; fp32 products, and the next
// segment's A and E are asked for before this one's are used.  Bound by the latency of those loads, 3 us a segment.
template <typename T> __global__ __launch_bounds__(CHUNK_THREADS) void merit_delta_join(DeltaParams p)
{
    constexpr int KEYS = MERIT_DELTA_MAX_KEYS;
    static_assert(CHUNK_THREADS / 64 * 16 == KEYS, "");
    __shared__ float s[KEYS][16];
    const int tiles = (p.Dv + 15) / 16, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15,
              quad = lane >> 4;
    const int64_t head = blockIdx.x / (uint32_t)tiles;
    const int c = (int)(blockIdx.x % (uint32_t)tiles) * 16 + l16, n = (tokens_of(p, head / p.H) + C - 1) / C;
    const int last = n > 0 ? (n - 1) / p.seg_chunks : 0, row = min(16 * wave + l16, p.Dk - 1), r0 = 16 * wave + 4 * quad;
    if (last < 2) return;
    const int64_t column = min(c, p.Dv - 1);                            // (what is not there is read somewhere, and not written)
    f32x4 a[KEYS / 16];
    float e[4];
    const int pitch = delta_pitch(p);
    auto load = [&](int j) __attribute__((always_inline)) {
        const float *A = segment_through(p, j) + (head * p.Dk + row) * pitch, *E = segment_state(p, j + 1) + head * p.Dk * p.Dv + column;
#pragma unroll
        for (int i = 0; i < KEYS / 16; ++i) a[i] = *reinterpret_cast<const f32x4 *>(A + min(16 * i + 4 * quad, pitch - 4));
#pragma unroll
        for (int i = 0; i < 4; ++i) e[i] = E[(int64_t)min(r0 + i, p.Dk - 1) * p.Dv];
    };
    const float *first = segment_state(p, 1) + head * p.Dk * p.Dv + column;
    for (int r = tid >> 4; r < KEYS; r += CHUNK_THREADS / 16) s[r][l16] = r < p.Dk ? first[(int64_t)r * p.Dv] : 0.0f;
    load(1);
    __syncthreads();
    for (int j = 1; j < last; ++j) {
        f32x4 acc = {e[0], e[1], e[2], e[3]};
        f32x4 now[KEYS / 16];
#pragma unroll
        for (int i = 0; i < KEYS / 16; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) now[i][k] = 16 * i + 4 * quad + k < p.Dk ? a[i][k] : 0.0f;
        if (j + 1 < last) load(j + 1);
#pragma unroll
        for (int i = 0; i < KEYS / 16; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(now[i][k], s[16 * i + 4 * quad + k][l16], acc, 0, 0, 0);
        __syncthreads();
        float *to = segment_state(p, j + 1) + head * p.Dk * p.Dv + c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r0 + i < p.Dk) {
                s[r0 + i][l16] = acc[i];
                if (c < p.Dv) to[(int64_t)(r0 + i) * p.Dv] = acc[i];
            }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// one token
// ---------------------------------------------------------------------------
// Bound by memory: the state is read once and held in registers.  y = q.S_t = a q.S_{t-1} + (q.k) u, so both sums over the
// state's rows come from the one pass (512 states of 128 x 128: 16.2 us, 4.1 TB/s; 4 of 64 x 64: 6.5, the launch).  A workgroup
// has `lanes` vectors of V columns, NT / lanes threads share a column's rows.
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
    const float decay = p.g.data ? exp2_of(log2_decay(static_cast<const float *>(p.g.data)[b * p.g.s0 + h])) : 1.0f;
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
template <typename T, int KF, Leaves LEAVES> hipError_t chunks_of(const DeltaParams &p, int segments, hipStream_t s)
{
    constexpr int lds = ForwardLds<T, KF>::bytes;
    static_assert(lds + 256 <= 160 * 1024, "");
    const dim3 grid((unsigned)(p.B * p.H * p.slices), (unsigned)segments);
    if (p.wide_qk) merit_delta_chunks<T, KF, true, LEAVES><<<grid, CHUNK_THREADS, lds, s>>>(p);
    else merit_delta_chunks<T, KF, false, LEAVES><<<grid, CHUNK_THREADS, lds, s>>>(p);
    return hipGetLastError();
}
template <typename T, int KF> hipError_t forward_of(DeltaParams p, hipStream_t s)
{
    if (hipError_t e = prepare_of<T, KF>(p, s)) return e;
    if (p.segments > 1) {
        DeltaParams o = p;
        o.width = delta_width(p.B * p.H * (p.segments - 1), p.Dv, p.Dk);
        o.slices = delta_slices(o.width, p.Dv, p.Dk);
        if (hipError_t e = chunks_of<T, KF, SEGMENT>(o, p.segments - 1, s)) return e;
        if (p.segments > 2) {
            merit_delta_join<T><<<(unsigned)(p.B * p.H * ((p.Dv + 15) / 16)), CHUNK_THREADS, 0, s>>>(p);
            if (hipError_t e = hipGetLastError()) return e;
        }
    }
    p.width = delta_width(p.B * p.H * p.segments, p.Dv, 0);
    p.slices = delta_slices(p.width, p.Dv, 0);
    return p.states ? chunks_of<T, KF, KEPT>(p, p.segments, s) : chunks_of<T, KF, RESULTS>(p, p.segments, s);
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
