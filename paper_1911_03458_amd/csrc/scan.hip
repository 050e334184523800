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

template <int SPL, int LPC, bool PAD> __global__ __launch_bounds__(NT) void merit_scan_tiles(ScanParams p)
{
    using S = Shape<SPL, LPC>;
    __shared__ __align__(16) float bl[2][TT * S::NP], cl[2][TT * S::NP];
    const Where w = where<LPC>(p, p.chunks);
    const int n0 = w.lane * SPL;
    float A[SPL], h[SPL];
    bool ok[SPL];
    const int64_t hat = (w.b * p.D + w.d) * p.N + n0;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        ok[s] = w.in && (!PAD || n0 + s < p.N);
        A[s] = ok[s] ? p.A[(int64_t)w.d * p.N + n0 + s] * LOG2E : 0.0f;
        h[s] = ok[s] && p.h0 ? p.h0[hat + s] : 0.0f;
    }
    const float bias = w.in && p.dt_bias ? p.dt_bias[w.d] : 0.0f, skip = w.in && p.skip ? p.skip[w.d] : 0.0f;
    uint32_t xr[S::TPL], dr[S::TPL], zr[S::TPL] = {}, br[S::EB], cr[S::EB];
    auto fetch = [&](int tile) {
        load_rows<SPL, LPC>(p.x, p.type, w, tile, xr);
        load_rows<SPL, LPC>(p.dt, p.type, w, tile, dr);
        if (p.z.data) load_rows<SPL, LPC>(p.z, p.type, w, tile, zr);
        load_states<SPL, LPC>(p.Bm, p, w, tile, br);
        load_states<SPL, LPC>(p.Cm, p, w, tile, cr);
    };
    if (w.tile0 < w.tend) fetch(w.tile0);
    for (int tile = w.tile0; tile < w.tend; ++tile) {
        float *bt = bl[tile & 1], *ct = cl[tile & 1];
        stage_states<SPL, LPC>(bt, p, w, tile, br);
        stage_states<SPL, LPC>(ct, p, w, tile, cr);
        float x[S::TPL], z[S::TPL], dt[S::TPL], dx[S::TPL], y[S::TPL];
        values(xr, p.type, x);
        values(zr, p.type, z);
        values(dr, p.type, dt);
#pragma unroll
        for (int i = 0; i < S::TPL; ++i) {
            const bool in = tile * TT + i * LPC + w.lane < w.n;
            const float v = dt[i] + bias;
            dt[i] = in ? (p.softplus ? softplusf(v) : v) : 0.0f;
            dx[i] = in ? dt[i] * x[i] : 0.0f;
            y[i] = 0.0f;
        }
        fetch(min(tile + 1, w.tend - 1));
        lds_barrier();
        if (p.states && w.in) {
            float *o = p.states + ((w.b * p.tiles + tile) * p.D + w.d) * p.N + n0;
#pragma unroll
            for (int s = 0; s < SPL; ++s)
                if (ok[s]) o[s] = h[s];
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const float dtv = from_lane<LPC>(dt[t / LPC], t % LPC), dxv = from_lane<LPC>(dx[t / LPC], t % LPC);
            float Bv[SPL], Cv[SPL], acc = 0.0f;
            read_states<SPL>(bt + t * S::NP + n0, Bv);
            read_states<SPL>(ct + t * S::NP + n0, Cv);
#pragma unroll
            for (int s = 0; s < SPL; ++s) {
                h[s] = fmaf(__builtin_amdgcn_exp2f(dtv * A[s]), h[s], dxv * Bv[s]);
                if (PAD && !ok[s]) h[s] = 0.0f;            // (an infinite input: 0 times it)
                acc = fmaf(h[s], Cv[s], acc);
            }
            acc = sum_channel<LPC>(acc);
            if (LPC == 1 || w.lane == t % LPC) y[t / LPC] = acc;
        }
        if (w.in) {
#pragma unroll
            for (int i = 0; i < S::TPL; ++i) {
                const int t = tile * TT + i * LPC + w.lane;
                float v = p.skip ? fmaf(skip, x[i], y[i]) : y[i];         // (absent: not 0 times an infinite x)
                if (p.z.data) v *= siluf(z[i]);
                if (t < p.L) store_el(p.y.data, p.type, w.b * p.y.s0 + t * p.y.s1 + w.d, t < w.n ? v : 0.0f);
            }
        }
    }
    if (!w.in) return;
    for (int64_t t = (int64_t)max(w.tend, w.tile0) * TT + w.lane; t < min((int64_t)w.tile1 * TT, p.L); t += LPC)
        store_el(p.y.data, p.type, w.b * p.y.s0 + t * p.y.s1 + w.d, 0.0f);
    if (p.h_last && w.chunk == p.chunks - 1) {
#pragma unroll
        for (int s = 0; s < SPL; ++s)
            if (ok[s]) p.h_last[hat + s] = h[s];
    }
}

template <int SPL, int LPC, bool PAD> __global__ __launch_bounds__(NT) void merit_scan_token(ScanParams p)
{
    const int64_t id = (int64_t)blockIdx.x * NT + threadIdx.x, row = id / LPC;
    const int lane = (int)id & (LPC - 1), n0 = lane * SPL;
    const bool in = row < p.B * p.D;
    const int64_t b = in ? row / p.D : 0;
    const int d = in ? (int)(row - b * p.D) : 0, g = d / p.Dg;
    const int64_t hat = (b * p.D + d) * p.N + n0;
    const float v = load_el(p.dt.data, p.type, b * p.dt.s0 + d) + (p.dt_bias ? p.dt_bias[d] : 0.0f);
    const float x = load_el(p.x.data, p.type, b * p.x.s0 + d), z = p.z.data ? load_el(p.z.data, p.type, b * p.z.s0 + d) : 0.0f;
    const float dt = p.softplus ? softplusf(v) : v, dx = dt * x;
    float acc = 0.0f;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        if (!in || (PAD && n0 + s >= p.N)) continue;
        const float a = __builtin_amdgcn_exp2f(dt * p.A[(int64_t)d * p.N + n0 + s] * LOG2E);
        const float h = fmaf(a, p.h0[hat + s], dx * load_el(p.Bm.data, p.type, b * p.Bm.s0 + (int64_t)g * p.N + n0 + s));
        p.h_last[hat + s] = h;
        acc = fmaf(h, load_el(p.Cm.data, p.type, b * p.Cm.s0 + (int64_t)g * p.N + n0 + s), acc);
    }
    acc = sum_channel<LPC>(acc);
    if (!in || lane != 0) return;
    float y = p.skip ? fmaf(p.skip[d], x, acc) : acc;
    if (p.z.data) y *= siluf(z);
    store_el(p.y.data, p.type, b * p.y.s0 + d, y);
}

struct Forward {
    const ScanParams &p;
    hipStream_t s;
    template <int SPL, int LPC, bool PAD> hipError_t run()
    {
        merit_scan_tiles<SPL, LPC, PAD><<<(unsigned)(p.B * p.chunks * p.G * p.ctiles), NT, 0, s>>>(p);
        return hipGetLastError();
    }
};
struct Token {
    const ScanParams &p;
    hipStream_t s;
    template <int SPL, int LPC, bool PAD> hipError_t run()
    {
        merit_scan_token<SPL, LPC, PAD><<<(unsigned)((p.B * p.D * LPC + NT - 1) / NT), NT, 0, s>>>(p);
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_scan(const ScanParams &p, hipStream_t s) { return by_states(p.N, Forward{p, s}); }
hipError_t launch_scan_step(const ScanParams &p, hipStream_t s) { return by_states(p.N, Token{p, s}); }

}  // namespace merit
