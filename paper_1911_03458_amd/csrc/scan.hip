// Selective state space scan, forward and for a single token:
//     s = softplus(dt + dt_bias)                                     (or dt + dt_bias)
//     h_t[d,n] = exp(s A[d,n]) h_{t-1}[d,n] + s x B_t[n]
//     y[t,d]   = (sum_n C_t[n] h_t[d,n] + skip[d] x) silu(z)
// Per state and token an exponential, two products, two multiply-adds: bound by the vector ALUs at 16 states (4 tensors of
// 2 bytes a channel and token against 16 exponentials), by memory below about 8.
// A lane has four states of a channel, N / 4 lanes a channel, 256 threads 1024 / N channels of one sequence; tokens go in
// tiles of 16.  Of a tile a lane loads x, dt and z of every N / 4-th token, so that steps and gates are computed once; a
// token's values reach the channel's other lanes inside the multiplying instructions (DPP).  B and C of a tile, the same
// for all channels, are staged in LDS as fp32.
#include "scan.h"

namespace merit {

using namespace scan;

namespace {

// WHAT a launch leaves: the results; the results and the states before every tile; of every chunk but the last the state
// that it adds (from a state of 0) and the sum of its steps, from which the next launch's chunks find their first states
enum { RESULTS, KEEP_STATES, CHUNK_STATES };

template <typename T, int SPL, int LPC, bool PAD, int WHAT> __global__ __launch_bounds__(NT) void merit_scan_tiles(ScanParams p)
{
    using S = Shape<SPL, LPC>;
    constexpr bool KEEP = WHAT == KEEP_STATES, SUMS = WHAT == CHUNK_STATES;
    __shared__ __align__(16) float bl[2][TT * S::NP], cl[SUMS ? 1 : 2][SUMS ? 4 : TT * S::NP];
    const Where w = where<LPC>(p, 0, SUMS ? p.chunks - 1 : p.chunks);
    const int n0 = w.lane * SPL;
    float A[SPL], h[SPL];
    bool ok[SPL];
    const int64_t hat = (w.b * p.D + w.d) * p.N + n0;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        ok[s] = !PAD || n0 + s < p.N;
        A[s] = ok[s] ? p.A[(int64_t)w.d * p.N + n0 + s] * LOG2E : 0.0f;
        h[s] = !SUMS && ok[s] && p.h0 ? p.h0[hat + s] : 0.0f;
    }
    float steps = 0.0f;
    if (!SUMS) through_chunks<SPL>(p, w, n0, A, ok, h, 0, w.chunk, 1);
    const float bias = p.dt_bias ? p.dt_bias[w.d] : 0.0f, skip = p.skip ? p.skip[w.d] : 0.0f;
    const Walk xw = walk_rows<T>(p.x, w), dw = walk_rows<T>(p.dt, w), zw = p.z.data ? walk_rows<T>(p.z, w) : xw,
               yw = walk_rows<T>(p.y, w), bw = walk_states<T, S::NP>(p.Bm, p, w), cw = walk_states<T, S::NP>(p.Cm, p, w);

    // Two tiles in flight: a tile's arithmetic is over before a load of it comes back
    struct Raw {
        raw_t<T> x[S::TPL], dt[S::TPL], z[S::TPL], b[S::EB], c[S::EB];
    };
    Raw even, odd;
    auto fetch = [&](Raw &r, int tile, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        load_walk<T, WHOLE>(xw, tile, S::LQ, w.tok, w.n - 1, r.x);
        load_walk<T, WHOLE>(dw, tile, S::LQ, w.tok, w.n - 1, r.dt);
        if (!SUMS) load_walk<T, WHOLE>(zw, tile, S::LQ, w.tok, w.n - 1, r.z);
        const int first = ((int)threadIdx.x & (TT * S::NP - 1)) / S::NP;
        load_walk<T, WHOLE>(bw, tile, NT / S::NP, first, w.n - 1, r.b);
        if (!SUMS) load_walk<T, WHOLE>(cw, tile, NT / S::NP, first, w.n - 1, r.c);
    };
    float out[S::TPL];                          // results of the tile before
    // all: this tile and the one after the next are whole
    auto run = [&](Raw &r, float *bt, float *ct, int tile, auto all) {
        constexpr bool ALL = decltype(all)::value;
        stage_states<T, SPL, LPC>(bt, p, w, tile, r.b);
        if constexpr (!SUMS) stage_states<T, SPL, LPC>(ct, p, w, tile, r.c);
        float x[S::TPL], z[S::TPL], dt[S::TPL], dx[S::TPL], y[S::TPL];
        values<T>(r.x, x);
        if constexpr (!SUMS) values<T>(r.z, z);
        values<T>(r.dt, dt);
#pragma unroll
        for (int i = 0; i < S::TPL; ++i) {
            const bool in = ALL || tile * TT + i * S::LQ + w.tok < w.n;
            const float v = dt[i] + bias;
            dt[i] = in ? (p.softplus ? softplusf(v) : v) : 0.0f;
            dx[i] = in ? dt[i] * x[i] : 0.0f;
            steps += dt[i];
        }
        if (!SUMS && tile > w.tile0) store_walk<T, true>(yw, tile - 1, S::LQ, w.tok, p.L, out);
        if (KEEP) {
            float *o = p.states + ((w.b * p.tiles + tile) * p.D + w.d) * p.N + n0;
#pragma unroll
            for (int s = 0; s < SPL; ++s)
                if (!PAD || ok[s]) o[s] = h[s];
        }
        fetch(r, ALL ? tile + 2 : min(tile + 2, w.tend - 1), all);
        lds_barrier();
        // Four tokens at a time; what needs LDS or an exponential is asked for four tokens ahead
        float Bv[2][4][SPL], Cv[2][4][SPL], a[2][4][SPL];
        auto ahead = [&](int k) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int t = 4 * k + u;
                read_states<SPL>(bt + t * S::NP + n0, Bv[k & 1][u]);
                if (!SUMS) read_states<SPL>(ct + t * S::NP + n0, Cv[k & 1][u]);
                const float dtv = from_lane<S::LQ>(dt[t / S::LQ], t % S::LQ);
#pragma unroll
                for (int s = 0; s < SPL; ++s) a[k & 1][u][s] = __builtin_amdgcn_exp2f(dtv * A[s]);
            }
        };
        ahead(0);
#pragma unroll
        for (int k = 0; k < TT / 4; ++k) {
            __builtin_amdgcn_sched_barrier(0);
            if (k + 1 < TT / 4) ahead(k + 1);
            float acc[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int t = 4 * k + u;
                const float dxv = from_lane<S::LQ>(dx[t / S::LQ], t % S::LQ);
                acc[u] = 0.0f;
#pragma unroll
                for (int s = 0; s < SPL; ++s) {
                    h[s] = fmaf(a[k & 1][u][s], h[s], dxv * Bv[k & 1][u][s]);
                    if (PAD && !ok[s]) h[s] = 0.0f;            // (an infinite input: 0 times it)
                    if (!SUMS) acc[u] = fmaf(h[s], Cv[k & 1][u][s], acc[u]);
                }
            }
            if (!SUMS) sum_to_tokens<LPC>(acc, y + 4 * k / S::LQ);
        }
        if (SUMS) return;
#pragma unroll
        for (int i = 0; i < S::TPL; ++i) {
            if (p.skip) y[i] = fmaf(skip, x[i], y[i]);          // (absent: not 0 times an infinite x)
            if (p.z.data) y[i] *= siluf(z[i]);
            out[i] = ALL || tile * TT + i * S::LQ + w.tok < w.n ? y[i] : 0.0f;
        }
    };
    if (w.tile0 < w.tend) {
        fetch(even, w.tile0, std::false_type{});
        fetch(odd, min(w.tile0 + 1, w.tend - 1), std::false_type{});
        const int whole = min(w.tend, w.n / TT);                // tiles before this one are whole
        int tile = w.tile0;
        for (; tile + 3 < whole; tile += 2) {
            run(even, bl[0], cl[0], tile, std::true_type{});
            run(odd, bl[1], cl[SUMS ? 0 : 1], tile + 1, std::true_type{});
        }
        for (; tile < w.tend; tile += 2) {
            run(even, bl[0], cl[0], tile, std::false_type{});
            if (tile + 1 < w.tend) run(odd, bl[1], cl[SUMS ? 0 : 1], tile + 1, std::false_type{});
        }
        if (!SUMS) store_walk<T, false>(yw, w.tend - 1, S::LQ, w.tok, p.L, out);
    }
    if (SUMS) {
        const int64_t at = (w.b * p.chunks + w.chunk) * p.D + w.d;
        steps = sum_channel<S::LQ>(steps);      // (a channel's further quads have the same tokens)
        if (w.lane == 0) p.chunk_dt[at] = steps;
#pragma unroll
        for (int s = 0; s < SPL; ++s)
            if (ok[s]) p.chunk_h[at * p.N + n0 + s] = h[s];
        return;
    }
    for (int64_t t = (int64_t)max(w.tend, w.tile0) * TT + w.lane; t < min((int64_t)w.tile1 * TT, p.L); t += LPC)
        static_cast<T *>(p.y.data)[w.b * p.y.s0 + t * p.y.s1 + w.d] = (T)0.0f;
    if (p.h_last && w.chunk == p.chunks - 1) {
#pragma unroll
        for (int s = 0; s < SPL; ++s)
            if (ok[s]) p.h_last[hat + s] = h[s];
    }
}

template <typename T> __device__ __forceinline__ float load_el(const void *base, int64_t at) { return (float)static_cast<const T *>(base)[at]; }

// One token: the state is read and written once, 8 bytes a state, and that is what bounds it (32 x 2048 channels, 16 states: 9 MB).
// Every load goes out before the first value is used; lanes without a channel or a state read what their neighbours do.
template <typename T, int SPL, int LPC, bool PAD> __global__ __launch_bounds__(NT) void merit_scan_token(ScanParams p)
{
    const int64_t id = (int64_t)blockIdx.x * NT + threadIdx.x, rows = p.B * p.D, row = min(id / LPC, rows - 1);
    const int lane = (int)threadIdx.x & (LPC - 1), n0 = lane * SPL;
    const bool in = id / LPC < rows;
    const uint32_t b = (uint32_t)((uint64_t)row / (uint32_t)p.D);
    const int d = (int)(row - (int64_t)b * p.D), g = d / p.Dg;
    float A[SPL], h[SPL], Bv[SPL], Cv[SPL];
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        const int n = PAD ? min(n0 + s, p.N - 1) : n0 + s;
        A[s] = p.A[(int64_t)d * p.N + n];
        h[s] = p.h0[row * p.N + n];
        Bv[s] = load_el<T>(p.Bm.data, b * p.Bm.s0 + (int64_t)g * p.N + n);
        Cv[s] = load_el<T>(p.Cm.data, b * p.Cm.s0 + (int64_t)g * p.N + n);
    }
    const float x = load_el<T>(p.x.data, b * p.x.s0 + d), raw = load_el<T>(p.dt.data, b * p.dt.s0 + d);
    const float z = p.z.data ? load_el<T>(p.z.data, b * p.z.s0 + d) : 0.0f;
    const float bias = p.dt_bias ? p.dt_bias[d] : 0.0f, skip = p.skip ? p.skip[d] : 0.0f;
    const float v = raw + bias, dt = p.softplus ? softplusf(v) : v, dx = dt * x;
    float acc = 0.0f;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        h[s] = fmaf(__builtin_amdgcn_exp2f(dt * (A[s] * LOG2E)), h[s], dx * Bv[s]);
        if (!PAD || n0 + s < p.N) acc = fmaf(h[s], Cv[s], acc);
    }
    acc = sum_channel<LPC>(acc);
    if (!in) return;
    float y = p.skip ? fmaf(skip, x, acc) : acc;
    if (p.z.data) y *= siluf(z);
    if (lane == 0) static_cast<T *>(p.y.data)[b * p.y.s0 + d] = (T)y;
    if (!PAD) store_states<SPL>(p.h_last + row * p.N + n0, h);
    else
#pragma unroll
        for (int s = 0; s < SPL; ++s)
            if (n0 + s < p.N) p.h_last[row * p.N + n0 + s] = h[s];
}

template <typename T> struct Forward {
    const ScanParams &p;
    hipStream_t s;
    template <int SPL, int LPC, bool PAD> hipError_t run()
    {
        const unsigned per = (unsigned)(p.B * p.G * p.ctiles);
        if (p.chunks > 1) merit_scan_tiles<T, SPL, LPC, PAD, CHUNK_STATES><<<per * (p.chunks - 1), NT, 0, s>>>(p);
        if (p.states) merit_scan_tiles<T, SPL, LPC, PAD, KEEP_STATES><<<per * p.chunks, NT, 0, s>>>(p);
        else merit_scan_tiles<T, SPL, LPC, PAD, RESULTS><<<per * p.chunks, NT, 0, s>>>(p);
        return hipGetLastError();
    }
};
template <typename T> struct Token {
    const ScanParams &p;
    hipStream_t s;
    template <int SPL, int LPC, bool PAD> hipError_t run()
    {
        merit_scan_token<T, SPL, LPC, PAD><<<(unsigned)((p.B * p.D * LPC + NT - 1) / NT), NT, 0, s>>>(p);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_scan(const ScanParams &p, hipStream_t s)
{
    if (p.type == MERIT_BF16) return by_states(p.N, Forward<bf16_t>{p, s});
    return p.type == MERIT_F16 ? by_states(p.N, Forward<f16_t>{p, s}) : by_states(p.N, Forward<float>{p, s});
}
hipError_t launch_scan_step(const ScanParams &p, hipStream_t s)
{
    if (p.type == MERIT_BF16) return by_states(p.N, Token<bf16_t>{p, s});
    return p.type == MERIT_F16 ? by_states(p.N, Token<f16_t>{p, s}) : by_states(p.N, Token<float>{p, s});
}
// (defined in the sources of their types)
hipError_t launch_scan_backward(const ScanParams &p, hipStream_t s)
{
    if (p.type == MERIT_BF16) return scan_backward_of<bf16_t>(p, s);
    return p.type == MERIT_F16 ? scan_backward_of<f16_t>(p, s) : scan_backward_of<float>(p, s);
}

}  // namespace merit
