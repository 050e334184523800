// Selective state space scan, backward.  With dy' = dy silu(z) and a_t = exp(s_t A):
//     l_t = C_t dy'_t + a_{t+1} l_{t+1}                    the adjoint of h_t, from the last token to the first
//     dB_t[n] = sum_d l_t s x,    dC_t[n] = sum_d dy'_t h_t        (sums over the channels of a group)
//     u = sum_n l_t B_t,  q[n] = l_t a_t h_{t-1},  ds = u x + sum_n q A,  dx = u s + skip dy'
//     ddt = ds sigmoid(dt + dt_bias),  dA[n] = sum_{b,t} q s,  dz = dy (C_t h_t + skip x) silu'(z)
// Tiles of 16 tokens from the last to the first; a tile starts from the state that the forward pass kept before it, so the
// states of its tokens are computed once more and stay, the decays in registers, the states in LDS.  dB and dC are sums over
// channels, which are lanes: the 16 tokens' values of a state are added across lanes so that every halving of the lanes
// halves the values too (15 exchanges for 16 sums of 16 lanes), then wavefronts through LDS, then workgroups through
// memory in a second launch, in a fixed order.
// Bound by the vector ALUs: a state and token take an exponential, 13 plain operations and two sums across lanes of 15/16 of
// an exchange and an addition each, about 51 cycles a wavefront and SIMD: 190 us for 8x2048x2048 and 16 states.  Measured there
// (bfloat16, gated): 531 us, in two chunks a sequence with 90 us for their first adjoints; 16 us for the sums of dB and dC and
// 5 us for those of dA.  (Two workgroups a compute unit is what registers and LDS allow at 9 to 16 states; a wait of one has but
// the other to fill it.  At 3 to 8 states registers allow one, 270 to 348 of them, and from 17 on LDS does, 88 or 112 KB.)
#pragma once
#include "merit_internal.h"
#include "scan.h"

namespace merit {

using namespace scan;

namespace {

// lanes whose bit BIT is 0: the sum of `lo` over the two lanes that differ in it; the others: the sum of `hi`
template <int BIT> __device__ __forceinline__ float halve(float lo, float hi)
{
    if constexpr (BIT >= 4) {
        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
        u32x2 r;
        const unsigned a = __builtin_bit_cast(unsigned, lo), b = __builtin_bit_cast(unsigned, hi);
        if constexpr (BIT == 5) r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(a, b, false, false));
        else r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(a, b, false, false));
        const unsigned u = r.x, v = r.y;        // (as values: a bit cast of a vector's element takes its first)
        return __builtin_bit_cast(float, u) + __builtin_bit_cast(float, v);
    } else {
        static_assert(BIT == 2 || BIT == 3, "");
        const int a = __builtin_bit_cast(int, lo), b = __builtin_bit_cast(int, hi);
        int o;
        if constexpr (BIT == 3) {       // row_ror:8 into the lower, then the upper eight lanes of sixteen
            o = __builtin_amdgcn_update_dpp(0, a, 0x128, 0xF, 0x3, false);
            o = __builtin_amdgcn_update_dpp(o, b, 0x128, 0xF, 0xC, false);
        } else {                        // row_ror:12 into the even quads, row_ror:4 into the odd ones
            o = __builtin_amdgcn_update_dpp(0, a, 0x12C, 0xF, 0x5, false);
            o = __builtin_amdgcn_update_dpp(o, b, 0x124, 0xF, 0xA, false);
        }
        return ((threadIdx.x >> BIT) & 1 ? hi : lo) + __builtin_bit_cast(float, o);
    }
}

// Values of the 16 tokens summed over the lanes of a wavefront that have the same state (all but the lowest log2 LPC lane
// bits): four tokens at a time over the highest two of these bits, the four results over the others.  The lane keeps the
// sums of KEEP tokens, token(0), ...
template <int LPC> struct Sums {
    static constexpr int KEEP = LPC <= 4 ? 1 : LPC / 4;
    static __device__ __forceinline__ int token(int j)
    {
        const int lane = threadIdx.x, k = LPC <= 4 ? (lane >> 2) & 3 : LPC == 8 ? ((lane >> 2) & 2) + j : j;
        return 4 * k + ((lane >> 4) & 3);
    }
    static __device__ __forceinline__ float of_four(float a, float b, float c, float d)
    {
        return halve<4>(halve<5>(a, c), halve<5>(b, d));
    }
    static __device__ __forceinline__ void of_all(float (&v)[4])
    {
        if constexpr (LPC <= 8) {
            v[0] = halve<3>(v[0], v[2]);
            v[1] = halve<3>(v[1], v[3]);
        }
        if constexpr (LPC <= 4) v[0] = halve<2>(v[0], v[1]);
        if constexpr (LPC <= 2) v[0] += lane_xor<1>(v[0]);
        if constexpr (LPC <= 1) v[0] += lane_xor<0>(v[0]);
    }
    // of the lanes that hold the same sum, the one that writes it
    static __device__ __forceinline__ bool writes() { return LPC >= 4 || (threadIdx.x & (3 & ~(LPC - 1))) == 0; }
};

// LDS of a workgroup: B and C of a tile, the wavefronts' sums for dB and dC, the states of the tile's tokens, zeros in the place
// of B and C
template <int SPL, int LPC> constexpr int back_lds()
{
    return (4 * TT * SPL * LPC + NT / 64 * TT * 2 * SPL * LPC + TT * NT * SPL) * 4;
}

// Two wavefronts a SIMD (a lone one issues plain arithmetic at half the rate) for 9 to 16 states, so 256 registers: the decays of
// a tile stay in registers, its states in LDS.  From 33 states on 5 to 8 registers spill.
template <typename T, int SPL, int LPC, bool PAD>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(LPC >= 4 ? 2 : 1, 2))) void merit_scan_back(ScanParams p)
{
    using S = Shape<SPL, LPC>;
    using Q = Sums<LPC>;
    extern __shared__ __align__(16) float lds[];
    float *const bl = lds, *const cl = bl + TT * S::NP, *const red = cl + TT * S::NP;
    float *const hl = red + NT / 64 * TT * 2 * S::NP + threadIdx.x * SPL;      // token t: t * NT * SPL further
    const Where w = where<LPC>(p, 0, p.chunks, threadIdx.x);
    const int n0 = w.lane * SPL, wave = threadIdx.x >> 6;
    // Lanes without a channel take part in the sums over channels: their x, dt and dy are zeros, and so are their B and C, of
    // which an infinity times 0 would be a NaN.  (An offset, of which the compiler sees what it is a multiple of: with a pointer
    // chosen 8x1024x1030 with one state took 111 us, with the offset 105.)
    constexpr int NONE = 2 * TT * S::NP + NT / 64 * TT * 2 * S::NP + TT * NT * SPL;
    for (int e = threadIdx.x; e < 2 * TT * S::NP; e += NT) lds[NONE + e] = 0.0f;
    const float *const bt = lds + (w.in ? 0 : NONE) + n0, *const ct = bt + TT * S::NP;
    float A2[SPL], dA[SPL], carry[SPL];                     // (A2: the exponentials are to the base 2)
    bool ok[SPL];
    const int64_t hat = (w.b * p.D + w.d) * p.N + n0;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        ok[s] = w.in && (!PAD || n0 + s < p.N);
        A2[s] = ok[s] ? p.A[(int64_t)w.d * p.N + n0 + s] * LOG2E : 0.0f;
        dA[s] = 0.0f;
        carry[s] = ok[s] && p.dh_last ? p.dh_last[hat + s] : 0.0f;     // a_{t+1} l_{t+1}
    }
    through_chunks<SPL>(p, w, n0, A2, ok, carry, p.chunks - 1, p.chunks - 1 - w.chunk, -1);
    const float bias = w.in && p.dt_bias ? p.dt_bias[w.d] : 0.0f, skip = w.in && p.skip ? p.skip[w.d] : 0.0f;
    float dskip = 0.0f, dbias = 0.0f;
    // behind the sequence's end every gradient is 0
    for (int64_t t = (int64_t)max(w.tend, w.tile0) * TT + w.lane; t < min((int64_t)w.tile1 * TT, p.L); t += LPC) {
        static_cast<T *>(p.dx.data)[w.b * p.dx.s0 + t * p.dx.s1 + w.d] = (T)0.0f;
        static_cast<T *>(p.ddt.data)[w.b * p.ddt.s0 + t * p.ddt.s1 + w.d] = (T)0.0f;
        if (p.z.data) static_cast<T *>(p.dz.data)[w.b * p.dz.s0 + t * p.dz.s1 + w.d] = (T)0.0f;
    }
    float *bc = p.part_bc + ((int64_t)(w.g * p.ctiles + w.ct) * p.B + w.b) * p.L * 2 * p.N;
    for (int64_t e = (int64_t)max(w.tend, w.tile0) * TT * 2 * p.N + threadIdx.x; e < min((int64_t)w.tile1 * TT, p.L) * 2 * p.N; e += NT) bc[e] = 0.0f;

    const Walk xw = walk_rows<T>(p.x, w), dw = walk_rows<T>(p.dt, w), yw = walk_rows<T>(p.dy, w),
               zw = p.z.data ? walk_rows<T>(p.z, w) : xw, bw = walk_states<T, S::NP>(p.Bm, p, w, threadIdx.x),
               cw = walk_states<T, S::NP>(p.Cm, p, w, threadIdx.x), dxw = walk_rows<T>(p.dx, w), ddw = walk_rows<T>(p.ddt, w),
               dzw = walk_rows<T>(p.dz, w);
    raw_t<T> xr[S::TPL], dr[S::TPL], yr[S::TPL], zr[S::TPL], br[S::EB], cr[S::EB];
    float hr[SPL];
    auto fetch = [&](int tile, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        load_walk<T, WHOLE>(xw, tile, S::LQ, w.tok, w.n - 1, xr);
        load_walk<T, WHOLE>(dw, tile, S::LQ, w.tok, w.n - 1, dr);
        load_walk<T, WHOLE>(yw, tile, S::LQ, w.tok, w.n - 1, yr);
        load_walk<T, WHOLE>(zw, tile, S::LQ, w.tok, w.n - 1, zr);
        const int first = ((int)threadIdx.x & (TT * S::NP - 1)) / S::NP;
        load_walk<T, WHOLE>(bw, tile, NT / S::NP, first, w.n - 1, br);
        load_walk<T, WHOLE>(cw, tile, NT / S::NP, first, w.n - 1, cr);
        const float *kept = p.states + ((w.b * p.tiles + tile) * p.D + w.d) * p.N;
#pragma unroll
        for (int s = 0; s < SPL; ++s) hr[s] = kept[PAD ? min(n0 + s, p.N - 1) : n0 + s];
    };
    // what a tile has computed: written while the next one is under way
    float ox[S::TPL], od[S::TPL], oz[S::TPL];
    auto write = [&](int tile) {
        // (lanes of a channel that is not there computed with zeros: they must not write over the one they stand for)
        if (w.in) {
            store_walk<T, false>(dxw, tile, S::LQ, w.tok, p.L, ox);
            store_walk<T, false>(ddw, tile, S::LQ, w.tok, p.L, od);
            if (p.z.data) store_walk<T, false>(dzw, tile, S::LQ, w.tok, p.L, oz);
        }
        constexpr int R = TT * 2 * S::NP;
#pragma unroll
        for (int i = 0; i < (R + NT - 1) / NT; ++i) {
            const int e = i * NT + (int)threadIdx.x, n = e % S::NP, k = e / S::NP;      // k = 2 t + (0: dB, 1: dC)
            const int64_t t = (int64_t)tile * TT + k / 2;
            if (e < R && n < p.N && t < p.L)
                bc[(t * 2 + (k & 1)) * p.N + n] = t < w.n ? (red[e] + red[e + R]) + (red[e + 2 * R] + red[e + 3 * R]) : 0.0f;
        }
    };
    auto run = [&](int tile, auto all) {
        constexpr bool ALL = decltype(all)::value;
        // of a token: x, step, step x, dy', the step's slope, dy silu'(z)
        float x[S::TPL], dt[S::TPL], dx[S::TPL], dy[S::TPL], slope[S::TPL], gz[S::TPL], y[S::TPL], in_[S::TPL], da_[S::TPL];
        values<T>(xr, x);
        values<T>(dr, dt);
        values<T>(yr, dy);
        values<T>(zr, gz);
        lds_barrier();              // (the tile before is done with bl and cl, and red is whole)
        if (tile + 1 < w.tend) write(tile + 1);
        stage_states<T, SPL, LPC>(bl, p, w, threadIdx.x, tile, br);
        stage_states<T, SPL, LPC>(cl, p, w, threadIdx.x, tile, cr);
        float h[SPL], hs[SPL], a[TT][SPL];
#pragma unroll
        for (int s = 0; s < SPL; ++s) h[s] = hs[s] = ok[s] ? hr[s] : 0.0f;
#pragma unroll
        for (int i = 0; i < S::TPL; ++i) {
            const bool in = w.in && (ALL || tile * TT + i * S::LQ + w.tok < w.n);
            const float v = dt[i] + bias, z = gz[i], g = dy[i];
            slope[i] = p.softplus ? sigmoidf(v) : 1.0f;
            dt[i] = in ? (p.softplus ? softplusf(v) : v) : 0.0f;
            dx[i] = in ? dt[i] * x[i] : 0.0f;
            dy[i] = in ? (p.z.data ? g * siluf(z) : g) : 0.0f;
            gz[i] = in ? g * act_slope(z, MERIT_ACT_SILU) : 0.0f;
        }
        fetch(max(tile - 1, w.tile0), all);
        lds_barrier();
        // the tile's states once more, four tokens at a time; dC on the way
        float sums[SPL][4];
#pragma unroll
        for (int k = 0; k < TT / 4; ++k) {
            __builtin_amdgcn_sched_barrier(0);
            float acc[4], c4[SPL][4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int t = 4 * k + u;
                const float dtv = from_lane<S::LQ>(dt[t / S::LQ], t % S::LQ), dxv = from_lane<S::LQ>(dx[t / S::LQ], t % S::LQ);
                const float dyv = from_lane<S::LQ>(dy[t / S::LQ], t % S::LQ);
                float Bv[SPL], Cv[SPL];
                read_states<SPL>(bt + t * S::NP, Bv);
                read_states<SPL>(ct + t * S::NP, Cv);
                acc[u] = 0.0f;
#pragma unroll
                for (int s = 0; s < SPL; ++s) {
                    a[t][s] = __builtin_amdgcn_exp2f(dtv * A2[s]);
                    h[s] = fmaf(a[t][s], h[s], dxv * Bv[s]);
                    if (PAD && !ok[s]) h[s] = 0.0f;
                    acc[u] = fmaf(h[s], Cv[s], acc[u]);
                    c4[s][u] = h[s] * dyv;
                }
                write_states<SPL>(hl + t * NT * SPL, h);
            }
            sum_to_tokens<LPC>(acc, y + 4 * k / S::LQ);
#pragma unroll
            for (int s = 0; s < SPL; ++s) sums[s][k] = Q::of_four(c4[s][0], c4[s][1], c4[s][2], c4[s][3]);
        }
        auto leave = [&](int kind) {
#pragma unroll
            for (int s = 0; s < SPL; ++s) {
                Q::of_all(sums[s]);
                if (Q::writes())
#pragma unroll
                    for (int j = 0; j < Q::KEEP; ++j)
                        red[wave * TT * 2 * S::NP + (2 * Q::token(j) + kind) * S::NP + n0 + s] = sums[s][j];
            }
        };
        leave(1);
        // (what the way back needs again it makes again: kept from above it would be more than the registers hold)
#pragma unroll
        for (int i = 0; i < S::TPL; ++i) asm volatile("" : "+v"(dt[i]), "+v"(dx[i]), "+v"(dy[i])::"memory");
        // and back: the adjoint of the state
#pragma unroll
        for (int k = TT / 4 - 1; k >= 0; --k) {
            __builtin_amdgcn_sched_barrier(0);
            float u4[4], v4[4], b4[SPL][4];
#pragma unroll
            for (int u = 3; u >= 0; --u) {
                const int t = 4 * k + u;
                const float dtv = from_lane<S::LQ>(dt[t / S::LQ], t % S::LQ), dxv = from_lane<S::LQ>(dx[t / S::LQ], t % S::LQ);
                const float dyv = from_lane<S::LQ>(dy[t / S::LQ], t % S::LQ);
                float Bv[SPL], Cv[SPL];
                read_states<SPL>(bt + t * S::NP, Bv);
                read_states<SPL>(ct + t * S::NP, Cv);
                if (t) read_states<SPL>(hl + (t - 1) * NT * SPL, h);
                u4[u] = v4[u] = 0.0f;
#pragma unroll
                for (int s = 0; s < SPL; ++s) {
                    float l = fmaf(Cv[s], dyv, carry[s]);
                    if (PAD && !ok[s]) l = 0.0f;
                    u4[u] = fmaf(l, Bv[s], u4[u]);
                    carry[s] = a[t][s] * l;
                    float q = carry[s] * (t ? h[s] : hs[s]);
                    if (!ALL && tile * TT + t >= w.n) q = 0.0f;         // (behind the end: an infinite state times 0)
                    v4[u] = fmaf(q, A2[s], v4[u]);
                    dA[s] = fmaf(q, dtv, dA[s]);
                    b4[s][u] = l * dxv;
                }
            }
            sum_to_tokens<LPC>(u4, in_ + 4 * k / S::LQ);
            sum_to_tokens<LPC>(v4, da_ + 4 * k / S::LQ);
#pragma unroll
            for (int s = 0; s < SPL; ++s) sums[s][k] = Q::of_four(b4[s][0], b4[s][1], b4[s][2], b4[s][3]);
        }
        leave(0);
#pragma unroll
        for (int i = 0; i < S::TPL; ++i) {
            const bool in = ALL || tile * TT + i * S::LQ + w.tok < w.n;
            const float ds = fmaf(in_[i], x[i], da_[i] * (1.0f / LOG2E)) * slope[i], y0 = p.skip ? fmaf(skip, x[i], y[i]) : y[i];
            if (in) {
                dskip = fmaf(dy[i], x[i], dskip);
                dbias += ds;
            }
            ox[i] = in ? (p.skip ? fmaf(in_[i], dt[i], skip * dy[i]) : in_[i] * dt[i]) : 0.0f;
            od[i] = in ? ds : 0.0f;
            oz[i] = in ? gz[i] * y0 : 0.0f;
        }
    };
    if (w.tile0 < w.tend) {
        fetch(w.tend - 1, std::false_type{});
        const int whole = min(w.tend, w.n / TT);
        if (whole < w.tend) run(w.tend - 1, std::false_type{});
        for (int tile = whole - 1; tile >= w.tile0; --tile) run(tile, std::true_type{});
        lds_barrier();
        write(w.tile0);
    }
    if (p.dh0 && w.chunk == 0) {
#pragma unroll
        for (int s = 0; s < SPL; ++s)
            if (ok[s]) p.dh0[hat + s] = carry[s];
    }
    float *part = p.part_a + (w.b * p.chunks + w.chunk) * ((int64_t)p.D * p.N + 2 * p.D);
#pragma unroll
    for (int s = 0; s < SPL; ++s)
        if (ok[s]) part[(int64_t)w.d * p.N + n0 + s] = dA[s];
    dskip = sum_channel<S::LQ>(dskip);          // (a channel's further quads have the same tokens)
    dbias = sum_channel<S::LQ>(dbias);
    if (w.in && w.lane == 0) {
        part[(int64_t)p.D * p.N + w.d] = dskip;
        part[(int64_t)p.D * p.N + p.D + w.d] = dbias;
    }
}

// Of every chunk but the first: the adjoint of the state before it that its own tokens leave, and the sum of its steps
template <typename T, int SPL, int LPC, bool PAD> __global__ __launch_bounds__(NT) void merit_scan_back_chunks(ScanParams p)
{
    using S = Shape<SPL, LPC>;
    __shared__ __align__(16) float cl[2][TT * S::NP];
    const Where w = where<LPC>(p, 1, p.chunks - 1, threadIdx.x);
    const int n0 = w.lane * SPL;
    float A[SPL], carry[SPL], steps = 0.0f;
    bool ok[SPL];
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        ok[s] = !PAD || n0 + s < p.N;
        A[s] = ok[s] ? p.A[(int64_t)w.d * p.N + n0 + s] * LOG2E : 0.0f;
        carry[s] = 0.0f;
    }
    const float bias = p.dt_bias ? p.dt_bias[w.d] : 0.0f;
    const Walk dw = walk_rows<T>(p.dt, w), yw = walk_rows<T>(p.dy, w), zw = p.z.data ? walk_rows<T>(p.z, w) : yw,
               cw = walk_states<T, S::NP>(p.Cm, p, w, threadIdx.x);
    struct Raw {
        raw_t<T> dt[S::TPL], dy[S::TPL], z[S::TPL], c[S::EB];
    };
    Raw even, odd;
    auto fetch = [&](Raw &r, int tile, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        load_walk<T, WHOLE>(dw, tile, S::LQ, w.tok, w.n - 1, r.dt);
        load_walk<T, WHOLE>(yw, tile, S::LQ, w.tok, w.n - 1, r.dy);
        load_walk<T, WHOLE>(zw, tile, S::LQ, w.tok, w.n - 1, r.z);
        load_walk<T, WHOLE>(cw, tile, NT / S::NP, ((int)threadIdx.x & (TT * S::NP - 1)) / S::NP, w.n - 1, r.c);
    };
    auto run = [&](Raw &r, float *ct, int tile, auto all) {
        constexpr bool ALL = decltype(all)::value;
        stage_states<T, SPL, LPC>(ct, p, w, threadIdx.x, tile, r.c);
        float dt[S::TPL], dy[S::TPL], z[S::TPL];
        values<T>(r.dt, dt);
        values<T>(r.dy, dy);
        values<T>(r.z, z);
#pragma unroll
        for (int i = 0; i < S::TPL; ++i) {
            const bool in = ALL || tile * TT + i * S::LQ + w.tok < w.n;
            const float v = dt[i] + bias;
            dt[i] = in ? (p.softplus ? softplusf(v) : v) : 0.0f;
            dy[i] = in ? (p.z.data ? dy[i] * siluf(z[i]) : dy[i]) : 0.0f;
            steps += dt[i];
        }
        fetch(r, max(tile - 2, w.tile0), all);
        lds_barrier();
        float Cv[2][4][SPL], a[2][4][SPL];
        auto ahead = [&](int k) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int t = 4 * k + u;
                read_states<SPL>(ct + t * S::NP + n0, Cv[k & 1][u]);
                const float dtv = from_lane<S::LQ>(dt[t / S::LQ], t % S::LQ);
#pragma unroll
                for (int s = 0; s < SPL; ++s) a[k & 1][u][s] = __builtin_amdgcn_exp2f(dtv * A[s]);
            }
        };
        ahead(TT / 4 - 1);
#pragma unroll
        for (int k = TT / 4 - 1; k >= 0; --k) {
            __builtin_amdgcn_sched_barrier(0);
            if (k) ahead(k - 1);
#pragma unroll
            for (int u = 3; u >= 0; --u) {
                const int t = 4 * k + u;
                const float dyv = from_lane<S::LQ>(dy[t / S::LQ], t % S::LQ);
#pragma unroll
                for (int s = 0; s < SPL; ++s) {
                    carry[s] = a[k & 1][u][s] * fmaf(Cv[k & 1][u][s], dyv, carry[s]);
                    if (PAD && !ok[s]) carry[s] = 0.0f;
                }
            }
        }
    };
    if (w.tile0 < w.tend) {
        int tile = w.tend - 1;
        const int whole = min(w.tend, w.n / TT);
        fetch(even, tile, std::false_type{});
        fetch(odd, max(tile - 1, w.tile0), std::false_type{});
        if (tile >= whole) {                            // (the next two are fetched into the other order)
            run(even, cl[0], tile, std::false_type{});
            --tile;
            for (; tile > w.tile0; tile -= 2) {
                run(odd, cl[1], tile, std::true_type{});
                run(even, cl[0], tile - 1, std::true_type{});
            }
            if (tile == w.tile0) run(odd, cl[1], tile, std::true_type{});
        } else {
            for (; tile > w.tile0; tile -= 2) {
                run(even, cl[0], tile, std::true_type{});
                run(odd, cl[1], tile - 1, std::true_type{});
            }
            if (tile == w.tile0) run(even, cl[0], tile, std::true_type{});
        }
    }
    const int64_t at = (w.b * p.chunks + w.chunk) * p.D + w.d;
    steps = sum_channel<S::LQ>(steps);
    if (w.lane == 0) p.chunk_dt[at] = steps;
#pragma unroll
    for (int s = 0; s < SPL; ++s)
        if (ok[s]) p.chunk_h[at * p.N + n0 + s] = carry[s];
}

// dB, dC: the sums over a group's channel tiles, rounded once
template <typename T> __global__ __launch_bounds__(NT) void merit_scan_sum_bc(ScanParams p)
{
    const int64_t id = (int64_t)blockIdx.x * NT + threadIdx.x, per = (int64_t)p.B * p.L * 2 * p.N;
    const int g = (int)(id / per);
    if (g >= p.G) return;
    const int64_t e = id - g * per, row = e / (2 * p.N), b = row / p.L, t = row - b * p.L;
    const int k = (int)(e - row * 2 * p.N), n = k < p.N ? k : k - p.N;
    const float *in = p.part_bc + (int64_t)g * p.ctiles * per + e;
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < p.ctiles; ++i) s += in[i * per];
    const Rows &o = k < p.N ? p.dB : p.dC;
    static_cast<T *>(o.data)[b * o.s0 + t * o.s1 + (int64_t)g * p.N + n] = (T)s;
}

template <typename T> struct Backward {
    const ScanParams &p;
    hipStream_t s;
    template <int SPL, int LPC, bool PAD> hipError_t run()
    {
        if (p.chunks > 1)
            merit_scan_back_chunks<T, SPL, LPC, PAD><<<(unsigned)(p.B * (p.chunks - 1) * p.G * p.ctiles), NT, 0, s>>>(p);
        static std::atomic<int> raised;
        const hipError_t e = raise_lds_limit_once(reinterpret_cast<const void *>(merit_scan_back<T, SPL, LPC, PAD>), raised);
        if (e != hipSuccess) return e;
        merit_scan_back<T, SPL, LPC, PAD>
            <<<(unsigned)(p.B * p.chunks * p.G * p.ctiles), NT, back_lds<SPL, LPC>(), s>>>(p);
        return hipGetLastError();
    }
};

}  // namespace

template <typename T> hipError_t scan_backward_of(const ScanParams &p, hipStream_t s)
{
    if (p.B > 0) {
        const hipError_t e = by_states(p.N, Backward<T>{p, s});
        if (e != hipSuccess) return e;
        const int64_t count = (int64_t)p.G * p.B * p.L * 2 * p.N;
        if (count) merit_scan_sum_bc<T><<<(unsigned)((count + NT - 1) / NT), NT, 0, s>>>(p);
    }
    ReduceParams r = {};
    r.in = p.part_a;
    r.rows = p.B * p.chunks;
    r.pitch = (int64_t)p.D * p.N + 2 * p.D;
    r.nseg = 3;
    r.seg[0] = {p.dA, 0, (int64_t)p.D * p.N};
    r.seg[1] = {p.dskip, (int64_t)p.D * p.N, p.D};
    r.seg[2] = {p.ddt_bias, (int64_t)p.D * p.N + p.D, p.D};
    return launch_reduce_rows(r, s);
}

}  // namespace merit
