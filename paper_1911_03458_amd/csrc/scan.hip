// Selective state space scan, forward and for a single token:
//     s = softplus(dt + dt_bias)                                     (or dt + dt_bias)
//     h_t[d,n] = exp(s A[d,n]) h_{t-1}[d,n] + s x B_t[n]
//     y[t,d]   = (sum_n C_t[n] h_t[d,n] + skip[d] x) silu(z)
// Per state and token an exponential, two products, two multiply-adds: bound by the vector ALUs at 16 states (4 tensors of
// 2 bytes a channel and token against 16 exponentials), by memory below about 4.
// A lane has four states of a channel, N / 4 lanes a channel, 256 threads 1024 / N channels of one sequence; tokens go in
// tiles of 16.  Steps, gates and the movement of x, dt, z and y, once per token and channel, are the work of 256 threads more.
// A token's step reaches the channel's lanes inside the multiplying instruction (DPP); B and C of a tile, the same for all
// channels, are staged in LDS as fp32.
// Measured (bfloat16, gated, 16 states; traced launch by launch): 8x2048x2048 176 us (271 MB: 1.5 TB/s; 0.54 G states x tokens:
// 3.1 T/s, exponentials and plain operations alone would allow 7.9 T/s), 150 us a call where calls follow one another;
// 1x8191x2048 in 16 chunks 87 us and 58 us for the chunks' first states, 121 a call; a token of 32x2048 channels 4.3 us.
// Without the second half of the workgroup, its work done by the first: 235 us, and 104 + 64.
// (With one state the second half, 16 tokens of a tile a thread, spills 77 registers.)
#include "merit_internal.h"
#include "scan.h"

namespace merit {

using namespace scan;

namespace {

// WHAT a launch leaves: the results; the results and the states before every tile; of every chunk but the last the state
// that it adds (from a state of 0) and the sum of its steps, from which the next launch's chunks find their first states
enum { RESULTS, KEEP_STATES, CHUNK_STATES };

// LDS of a workgroup, in floats, twice each for alternating tiles: (step, step x) and sums of 16 tokens x CPB channels, B and C
template <int SPL, int LPC> struct Room {
    using S = Shape<SPL, LPC>;
    static constexpr int PITCH = S::CPB + 8;               // (lanes that read neighbouring tokens: other banks)
    static constexpr int TOKENS = TT * PITCH * 2, SUMS = TT * PITCH, STATES = TT * S::NP;
    static constexpr int BYTES = 4 * 2 * (TOKENS + SUMS + 2 * STATES);
};

// A workgroup is two halves.  The first 256 threads run the recurrence: they read steps, B and C from LDS and leave the tokens'
// sums there.  The other 256 do what is done once per token and channel -- loads from memory, steps, gates, results --
// a tile ahead of the first half and a tile behind it.  So a SIMD has a wavefront of either kind, and one's waits are the other's
// arithmetic; the recurrence itself has no loads from memory to wait for.
template <typename T, int SPL, int LPC, bool PAD, int WHAT> __global__ __launch_bounds__(2 * NT) void merit_scan_tiles(ScanParams p)
{
    using S = Shape<SPL, LPC>;
    using R = Room<SPL, LPC>;
    constexpr bool KEEP = WHAT == KEEP_STATES, SUMS = WHAT == CHUNK_STATES;
    extern __shared__ __align__(16) float lds[];
    float *const tokens = lds, *const sums = tokens + 2 * R::TOKENS, *const bl = sums + 2 * R::SUMS, *const cl = bl + 2 * R::STATES;
    Where w = where<LPC>(p, 0, SUMS ? p.chunks - 1 : p.chunks, (int)threadIdx.x & (NT - 1));
    const int count = max(0, w.tend - w.tile0);            // tiles; a step for each, one before and one after them

    if (threadIdx.x >= NT) {
        constexpr int IP = TT / LPC;                        // tokens of a tile that a thread has: first, first + LPC, ...
        const int thread = (int)threadIdx.x - NT, c = thread % S::CPB, first = thread / S::CPB;
        w.d = w.g * p.Dg + min(w.ct * S::CPB + c, p.Dg - 1);
        w.tok = first;
        const float bias = p.dt_bias ? p.dt_bias[w.d] : 0.0f, skip = p.skip ? p.skip[w.d] : 0.0f;
        const Walk xw = walk_rows<T>(p.x, w), dw = walk_rows<T>(p.dt, w), zw = p.z.data ? walk_rows<T>(p.z, w) : xw,
                   yw = walk_rows<T>(p.y, w), bw = walk_states<T, S::NP>(p.Bm, p, w, thread), cw = walk_states<T, S::NP>(p.Cm, p, w, thread);
        struct Raw {
            raw_t<T> x[IP], dt[IP], z[IP], b[S::EB], c[S::EB];
        };
        Raw raw[4];                                         // tiles i, i + 4, ...: from their loads to their results
        float steps = 0.0f;
        auto fetch = [&](Raw &r, int tile, auto whole) {
            constexpr bool WHOLE = decltype(whole)::value;
            const int state = (thread & (TT * S::NP - 1)) / S::NP;
            load_walk<T, WHOLE>(xw, tile, LPC, first, w.n - 1, r.x);
            load_walk<T, WHOLE>(dw, tile, LPC, first, w.n - 1, r.dt);
            if (!SUMS) load_walk<T, WHOLE>(zw, tile, LPC, first, w.n - 1, r.z);
            load_walk<T, WHOLE>(bw, tile, NT / S::NP, state, w.n - 1, r.b);
            if (!SUMS) load_walk<T, WHOLE>(cw, tile, NT / S::NP, state, w.n - 1, r.c);
        };
        // Step s: results of tile s - 2 (kept in `last`), tile s made ready from `now`, tile s + 2 asked for (into `last`).
        // all: these tiles are there and whole
        auto step = [&](int s, Raw &now, Raw &last, auto all) {
            constexpr bool ALL = decltype(all)::value;
            const int tile = w.tile0 + s;
            if (!SUMS && (ALL || s >= 2)) {
                float x[IP], z[IP], y[IP];
                values<T>(last.x, x);
                values<T>(last.z, z);
#pragma unroll
                for (int i = 0; i < IP; ++i) {
                    y[i] = sums[(s & 1) * R::SUMS + (first + i * LPC) * R::PITCH + c];
                    if (p.skip) y[i] = fmaf(skip, x[i], y[i]);          // (absent: not 0 times an infinite x)
                    if (p.z.data) y[i] *= siluf(z[i]);
                    if (!ALL && (tile - 2) * TT + first + i * LPC >= w.n) y[i] = 0.0f;
                }
                store_walk<T, ALL>(yw, tile - 2, LPC, first, p.L, y);
            }
            if (ALL || s < count) {
                float x[IP], dt[IP];
                values<T>(now.x, x);
                values<T>(now.dt, dt);
                float *const to = tokens + (s & 1) * R::TOKENS;
#pragma unroll
                for (int i = 0; i < IP; ++i) {
                    const bool in = ALL || tile * TT + first + i * LPC < w.n;
                    const float v = dt[i] + bias;
                    dt[i] = in ? (p.softplus ? softplusf(v) : v) : 0.0f;
                    steps += dt[i];
                    *reinterpret_cast<float2 *>(to + 2 * ((first + i * LPC) * R::PITCH + c)) = make_float2(dt[i], in ? dt[i] * x[i] : 0.0f);
                }
                stage_states<T, SPL, LPC>(bl + (s & 1) * R::STATES, p, w, thread, tile, now.b);
                if constexpr (!SUMS) stage_states<T, SPL, LPC>(cl + (s & 1) * R::STATES, p, w, thread, tile, now.c);
            }
            if (ALL) fetch(last, tile + 2, all);
            else if (count) fetch(last, min(tile + 2, w.tend - 1), all);
            lds_barrier();
        };
        if (count) {
            fetch(raw[0], w.tile0, std::false_type{});
            fetch(raw[1], min(w.tile0 + 1, w.tend - 1), std::false_type{});
        }
        const int total = count + 2, whole = min(w.tend, w.n / TT) - w.tile0;       // tiles 0 ... whole - 1 are whole
        step(0, raw[0], raw[2], std::false_type{});
        step(1, raw[1], raw[3], std::false_type{});
        int s = 2;
        for (; s + 5 < whole; s += 4) {
            step(s, raw[2], raw[0], std::true_type{});
            step(s + 1, raw[3], raw[1], std::true_type{});
            step(s + 2, raw[0], raw[2], std::true_type{});
            step(s + 3, raw[1], raw[3], std::true_type{});
        }
        for (; s < total; s += 4) {
            step(s, raw[2], raw[0], std::false_type{});
            if (s + 1 < total) step(s + 1, raw[3], raw[1], std::false_type{});
            if (s + 2 < total) step(s + 2, raw[0], raw[2], std::false_type{});
            if (s + 3 < total) step(s + 3, raw[1], raw[3], std::false_type{});
        }
        if (SUMS) {                                         // the chunk's steps, over the threads of a channel
            tokens[first * S::CPB + c] = steps;
            lds_barrier();
            if (first == 0) {
#pragma unroll
                for (int i = 1; i < LPC; ++i) steps += tokens[i * S::CPB + c];
                p.chunk_dt[(w.b * p.chunks + w.chunk) * p.D + w.d] = steps;
            }
        } else {
            for (int64_t t = (int64_t)max(w.tend, w.tile0) * TT + first; t < min((int64_t)w.tile1 * TT, p.L); t += LPC)
                static_cast<T *>(p.y.data)[w.b * p.y.s0 + t * p.y.s1 + w.d] = (T)0.0f;
        }
        return;
    }

    const int n0 = w.lane * SPL, c = (int)threadIdx.x / LPC;
    float A[SPL], h[SPL];
    bool ok[SPL];
    const int64_t hat = (w.b * p.D + w.d) * p.N + n0;
#pragma unroll
    for (int s = 0; s < SPL; ++s) {
        ok[s] = !PAD || n0 + s < p.N;
        A[s] = ok[s] ? p.A[(int64_t)w.d * p.N + n0 + s] * LOG2E : 0.0f;
        h[s] = !SUMS && ok[s] && p.h0 ? p.h0[hat + s] : 0.0f;
    }
    if (!SUMS) through_chunks<SPL>(p, w, n0, A, ok, h, 0, w.chunk, 1);
    lds_barrier();
    for (int i = 0; i < count; ++i) {
        const int tile = w.tile0 + i;
        const float *const bt = bl + (i & 1) * R::STATES + n0, *const ct = cl + (i & 1) * R::STATES + n0,
                    *const tt = tokens + (i & 1) * R::TOKENS + 2 * (w.tok * R::PITCH + c);
        float *const st = sums + (i & 1) * R::SUMS + w.tok * R::PITCH + c;
        if (KEEP) {
            float *o = p.states + ((w.b * p.tiles + tile) * p.D + w.d) * p.N + n0;
#pragma unroll
            for (int s = 0; s < SPL; ++s)
                if (!PAD || ok[s]) o[s] = h[s];
        }
        float dt[S::TPL], dx[S::TPL];
#pragma unroll
        for (int k = 0; k < S::TPL; ++k) {
            const float2 v = *reinterpret_cast<const float2 *>(tt + 2 * k * S::LQ * R::PITCH);
            dt[k] = v.x;
            dx[k] = v.y;
        }
        // Four tokens at a time; what needs LDS or an exponential is asked for four tokens ahead
        float Bv[2][4][SPL], Cv[2][4][SPL], a[2][4][SPL];
        auto ahead = [&](int k) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int t = 4 * k + u;
                read_states<SPL>(bt + t * S::NP, Bv[k & 1][u]);
                if (!SUMS) read_states<SPL>(ct + t * S::NP, Cv[k & 1][u]);
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
            float acc[4], y[4 / S::LQ];
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
            if (SUMS) continue;
            sum_to_tokens<LPC>(acc, y);
#pragma unroll
            for (int j = 0; j < 4 / S::LQ; ++j) st[(4 * k + j * S::LQ) * R::PITCH] = y[j];
        }
        lds_barrier();
    }
    lds_barrier();
    if (SUMS) lds_barrier();                                // (the other half adds up the steps)
    float *const out = SUMS ? p.chunk_h + ((w.b * p.chunks + w.chunk) * p.D + w.d) * p.N + n0
                            : p.h_last && w.chunk == p.chunks - 1 ? p.h_last + hat : nullptr;
    if (out)
#pragma unroll
        for (int s = 0; s < SPL; ++s)
            if (ok[s]) out[s] = h[s];
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
        const int64_t per = p.B * p.G * p.ctiles;
        if (p.chunks > 1) {
            const hipError_t e = launch<SPL, LPC, PAD, CHUNK_STATES>(per * (p.chunks - 1));
            if (e != hipSuccess) return e;
        }
        return p.states ? launch<SPL, LPC, PAD, KEEP_STATES>(per * p.chunks) : launch<SPL, LPC, PAD, RESULTS>(per * p.chunks);
    }
    template <int SPL, int LPC, bool PAD, int WHAT> hipError_t launch(int64_t blocks)
    {
        static std::atomic<int> raised;
        const auto kernel = merit_scan_tiles<T, SPL, LPC, PAD, WHAT>;
        hipError_t e = raise_lds_limit_once(reinterpret_cast<const void *>(kernel), raised);
        ScanParams q = p;
        for (int64_t at = 0; at < blocks && e == hipSuccess; at += SCAN_FORWARD_BLOCKS) {
            const int64_t rest = blocks - at;
            q.block0 = (uint32_t)at;
            kernel<<<(unsigned)(rest < SCAN_FORWARD_BLOCKS ? rest : SCAN_FORWARD_BLOCKS), 2 * NT, Room<SPL, LPC>::BYTES, s>>>(q);
            e = hipGetLastError();
        }
        return e;
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
