// Short causal convolution over tokens, channels last: k = (b, t, d | a),
//     M(x)[p,a] = x[b, t + a - (K-1), d]      (rows before the first: `init`, or 0)
//     M(w)[p,a] = w[d, a]
// reduced with the dot product, bias and activation on top: y = act(u).  Backward: du = dy act'(u),
//     dx[t] = sum_a w[a] du[t + K-1 - a],   dw[a] = sum_t du[t] x[t + a - (K-1)],   db = sum_t du[t].
// Bound by memory: 2 passes of the tensor forward, 3 backward.  A lane has four channels and walks down a strip of tokens
// with the window's rows, taps and sums in registers, so a row is read once per strip and its last K - 1 once more by the
// strip after it.  The gradients of taps and bias are summed over a workgroup's strips in LDS and over workgroups by a second
// launch, in a fixed order.
// Measured (bfloat16, K 4, SiLU): forward 8x2048x2048 30 us (134 MB: 4.5 TB/s), 3x4099x1536 17 us (76 MB: 4.4 TB/s); backward
// 8x2048x2048 51 us (201 MB: 4.0 TB/s; a copy of this size 6.0) and 5 us of sums; a token of 32x2048 channels 3.1 us: a launch.
#include "tokens.h"

namespace merit {

namespace {

constexpr int NT = 256;

struct Place {
    int64_t b, t0;
    int c;
    int64_t n;             // tokens of the sequence
    bool in;               // the strip is there
    bool own;              // so are the channels; a lane that has none does its wavefront's last ones again (and stores the same)
    int64_t strip;
    int sub, ct, row_lanes;
    int64_t row_block;
};
// 256 threads: ct (a power of two, at most 64) units of V channels x 256 / ct strips
template <int V> __device__ __forceinline__ Place place(const CconvParams &p)
{
    const int cu = p.D / V;
    Place q;
    q.ct = 1;
    while (q.ct < 64 && q.ct < cu) q.ct *= 2;
    q.row_lanes = NT / q.ct;
    const uint32_t tiles = (uint32_t)((cu + q.ct - 1) / q.ct);
    q.row_block = blockIdx.x / tiles;
    const int unit = (int)(blockIdx.x - (uint32_t)q.row_block * tiles) * q.ct + ((int)threadIdx.x & (q.ct - 1));
    q.sub = (int)threadIdx.x / q.ct;
    const int64_t s = q.row_block * q.row_lanes + q.sub;
    q.in = s < p.B * p.strips;
    q.own = q.in && unit < cu;
    q.b = q.in ? s / p.strips : 0;
    q.strip = s - q.b * p.strips;
    q.t0 = q.strip * p.strip;
    q.c = min(unit, cu - 1) * V;
    q.n = p.L;
    if (p.lens && q.in) q.n = min((int64_t)max(p.lens[q.b], 0), p.L);
    return q;
}

// row t of (init, x), t >= -(K-1)
template <typename T, int V, int K>
__device__ __forceinline__ vec_t<T, V> row_of(const CconvParams &p, const Place &q, int64_t t)
{
    if (t >= 0) return load_vec<T, V>(p.x.data, q.b * p.x.s0 + t * p.x.s1 + q.c);
    if (p.init.data) return load_vec<T, V>(p.init.data, q.b * p.init.s0 + (K - 1 + t) * p.init.s1 + q.c);
    return vec_t<T, V>{};
}

template <typename T, int V, int K>
__device__ __forceinline__ void load_taps(const CconvParams &p, int c, float (&w)[K][V], float (&b)[V])
{
    float flat[K * V];
    load_params<T>(p.w, (int64_t)c * K, 0.0f, flat);
    load_params<T>(p.b, c, 0.0f, b);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int a = 0; a < K; ++a) w[a][i] = flat[i * K + a];
}

// Strips run in batches of RB rows, two batches of loads in flight.  Loads and stores share one counter, so a load is waited
// for alone only where it is known how many loads and stores came after it: in a wavefront whose lanes all have a whole strip
// no load and no store stands under a condition.  Others (a sequence's end, channels that do not fill a wavefront) go row by row.
constexpr int RB = 4;
__device__ __forceinline__ bool whole_wavefront(bool lane_whole) { return __all(lane_whole) && __ballot(1) == ~0ull; }

template <typename T, int V, int K> __global__ __launch_bounds__(NT) void merit_cconv(CconvParams p)
{
    const Place q = place<V>(p);
    if (!q.in) return;
    float w[K][V], b[V], win[K][V];         // win[K-1]: the row of the current token
    load_taps<T, V, K>(p, q.c, w, b);
    const int64_t t1 = min(q.t0 + p.strip, q.n), t2 = min(q.t0 + p.strip, p.L);
    const int64_t yb = q.b * p.y.s0 + q.c;
    if (q.t0 < t1) {
#pragma unroll
        for (int j = 1; j < K; ++j) {
            const vec_t<T, V> v = row_of<T, V, K>(p, q, q.t0 - K + j);
#pragma unroll
            for (int i = 0; i < V; ++i) win[j][i] = at<T, V>(v, i);
        }
    }
    auto token = [&](const vec_t<T, V> &row) {      // one token: the window moves on, y of its last row
        vec_t<T, V> o;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float u = b[i];
#pragma unroll
            for (int a = 0; a < K - 1; ++a) {
                win[a][i] = win[a + 1][i];
                u = fmaf(w[a][i], win[a][i], u);
            }
            win[K - 1][i] = at<T, V>(row, i);
            u = fmaf(w[K - 1][i], win[K - 1][i], u);
            put<T, V>(o, i, apply_act(u, p.act));
        }
        return o;
    };
    if (whole_wavefront(t1 - q.t0 == p.strip)) {
        int64_t xa = q.b * p.x.s0 + q.t0 * p.x.s1 + q.c, ya = yb + q.t0 * p.y.s1;
        vec_t<T, V> v[2][RB];
        auto fetch = [&](vec_t<T, V>(&r)[RB]) {
#pragma unroll
            for (int k = 0; k < RB; ++k, xa += p.x.s1) r[k] = load_vec<T, V>(p.x.data, xa);
        };
        auto run = [&](vec_t<T, V>(&r)[RB], bool more) {
            vec_t<T, V> o[RB];
#pragma unroll
            for (int k = 0; k < RB; ++k) o[k] = token(r[k]);
            if (more) fetch(r);
#pragma unroll
            for (int k = 0; k < RB; ++k, ya += p.y.s1) store_vec<T, V>(p.y.data, ya, o[k]);
        };
        fetch(v[0]);
        fetch(v[1]);
        for (int k = 0; k + 2 < p.strip / RB; k += 2) {
            run(v[0], true);
            run(v[1], true);
        }
        run(v[0], false);
        run(v[1], false);
    } else {
        for (int64_t t = q.t0; t < t1; ++t)
            store_vec<T, V>(p.y.data, yb + t * p.y.s1, token(load_vec<T, V>(p.x.data, q.b * p.x.s0 + t * p.x.s1 + q.c)));
    }
    for (int64_t t = max(q.t0, q.n); t < t2; ++t) store_vec<T, V>(p.y.data, yb + t * p.y.s1, vec_t<T, V>{});
    if (K > 1 && p.fin.data && q.strip == 0 && q.own) {      // (every row is read before one is written: fin may be init)
        vec_t<T, V> v[K];
#pragma unroll
        for (int j = 0; j < K - 1; ++j) v[j] = row_of<T, V, K>(p, q, q.n - (K - 1) + j);
#pragma unroll
        for (int j = 0; j < K - 1; ++j) store_vec<T, V>(p.fin.data, q.b * p.fin.s0 + j * p.fin.s1 + q.c, v[j]);
    }
}

template <typename T, int V, int K> __global__ __launch_bounds__(NT) void merit_cconv_backward(CconvParams p)
{
    __shared__ float red[NT][V];
    const Place q = place<V>(p);
    float db[V], dw[K][V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        db[i] = 0.0f;
#pragma unroll
        for (int a = 0; a < K; ++a) dw[a][i] = 0.0f;
    }
    if (q.in) {
        float w[K][V], b[V], win[K][V], du[K][V];   // win[K-1], du[K-1]: of token s
        load_taps<T, V, K>(p, q.c, w, b);
        const int64_t t1 = min(q.t0 + p.strip, q.n), t2 = min(q.t0 + p.strip, p.L);
        const int64_t ob = q.b * p.dx.s0 + q.c, xb = q.b * p.x.s0 + q.c, yb = q.b * p.dy.s0 + q.c;
        if (q.t0 < t1) {
#pragma unroll
            for (int j = 1; j < K; ++j) {
                const vec_t<T, V> v = row_of<T, V, K>(p, q, q.t0 - K + j);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    win[j][i] = at<T, V>(v, i);
                    du[j][i] = 0.0f;
                }
            }
        }
        float none[V];
#pragma unroll
        for (int i = 0; i < V; ++i) none[i] = 0.0f;
        // token s: its u and du; `in`: it is there, `own`: it is the strip's; dx of the token K - 1 before it,
        // `more` added
        auto token = [&](const vec_t<T, V> &xrow, const vec_t<T, V> &yrow, bool in, bool own, const float (&more)[V]) {
            vec_t<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float u = b[i];
#pragma unroll
                for (int a = 0; a < K - 1; ++a) {
                    win[a][i] = win[a + 1][i];
                    du[a][i] = du[a + 1][i];
                    u = fmaf(w[a][i], win[a][i], u);
                }
                win[K - 1][i] = at<T, V>(xrow, i);
                u = fmaf(w[K - 1][i], win[K - 1][i], u);
                const float d = in ? at<T, V>(yrow, i) * act_slope(u, p.act) : 0.0f;
                du[K - 1][i] = d;
                if (own) {
                    db[i] += d;
#pragma unroll
                    for (int a = 0; a < K; ++a) dw[a][i] = fmaf(d, win[a][i], dw[a][i]);
                }
                float g = more[i];
#pragma unroll
                for (int a = 0; a < K; ++a) g = fmaf(w[a][i], du[K - 1 - a][i], g);
                put<T, V>(o, i, g);
            }
            return o;
        };
        // (the gradient of the last tokens kept: rows at the end of a sequence)
        if (whole_wavefront(t1 - q.t0 == p.strip && !p.dfin.data)) {
            const int64_t last = q.n - 1;
            auto rows = [&](int64_t s, vec_t<T, V> &x, vec_t<T, V> &y) {
                const int64_t r = min(s, last);
                x = load_vec<T, V>(p.x.data, xb + r * p.x.s1);
                y = load_vec<T, V>(p.dy.data, yb + r * p.dy.s1);
            };
            if constexpr (K > 1) {                      // the first K - 1 tokens finish no dx of the strip
                vec_t<T, V> x[K], y[K];
#pragma unroll
                for (int k = 0; k < K - 1; ++k) rows(q.t0 + k, x[k], y[k]);
#pragma unroll
                for (int k = 0; k < K - 1; ++k) token(x[k], y[k], q.t0 + k < q.n, true, none);
            }
            vec_t<T, V> x[2][RB], y[2][RB];
            int64_t s = q.t0 + K - 1, oa = ob + q.t0 * p.dx.s1;
            auto fetch = [&](int64_t from, vec_t<T, V>(&xr)[RB], vec_t<T, V>(&yr)[RB]) {
#pragma unroll
                for (int k = 0; k < RB; ++k) rows(from + k, xr[k], yr[k]);
            };
            auto run = [&](vec_t<T, V>(&xr)[RB], vec_t<T, V>(&yr)[RB], bool more) {
                vec_t<T, V> o[RB];
#pragma unroll
                for (int k = 0; k < RB; ++k) o[k] = token(xr[k], yr[k], s + k < q.n, s + k < t1, none);
                if (more) fetch(s + 2 * RB, xr, yr);
#pragma unroll
                for (int k = 0; k < RB; ++k, oa += p.dx.s1) store_vec<T, V>(p.dx.data, oa, o[k]);
                s += RB;
            };
            fetch(s, x[0], y[0]);
            fetch(s + RB, x[1], y[1]);
            for (int k = 0; k + 2 < p.strip / RB; k += 2) {
                run(x[0], y[0], true);
                run(x[1], y[1], true);
            }
            run(x[0], y[0], false);
            run(x[1], y[1], false);
        } else if (q.t0 < t1) {
            for (int64_t s = q.t0; s < t1 + K - 1; ++s) {
                const int64_t t = s - (K - 1);
                vec_t<T, V> xv{}, yv{};
                if (s < q.n) {
                    xv = load_vec<T, V>(p.x.data, xb + s * p.x.s1);
                    yv = load_vec<T, V>(p.dy.data, yb + s * p.dy.s1);
                }
                float more[V];
#pragma unroll
                for (int i = 0; i < V; ++i) more[i] = 0.0f;
                if (p.dfin.data && t >= q.t0 && t >= q.n - (K - 1)) {
                    const T *f = static_cast<const T *>(p.dfin.data) + q.b * p.dfin.s0 + (t - (q.n - (K - 1))) * p.dfin.s1 + q.c;
#pragma unroll
                    for (int i = 0; i < V; ++i) more[i] = (float)f[i];
                }
                const vec_t<T, V> o = token(xv, yv, s < q.n, s < t1, more);
                if (t < q.t0) continue;
                store_vec<T, V>(p.dx.data, ob + t * p.dx.s1, o);
            }
        }
        for (int64_t t = max(q.t0, q.n); t < t2; ++t) store_vec<T, V>(p.dx.data, ob + t * p.dx.s1, vec_t<T, V>{});
    }
    if (!p.dw && !p.db) return;
    float *out = p.part + q.row_block * (K + 1) * p.D;
    const bool unit_own = q.own;                // (the first strip of a workgroup is there)
#pragma unroll
    for (int a = 0; a <= K; ++a) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) red[threadIdx.x][i] = a < K ? dw[a < K ? a : 0][i] : db[i];
        __syncthreads();
        if (q.sub == 0 && unit_own) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float s = red[threadIdx.x][i];
                for (int k = 1; k < q.row_lanes; ++k) s += red[threadIdx.x + k * q.ct][i];
                // (taps of a channel side by side, as dweight has them; the bias' sums behind them)
                out[a < K ? (int64_t)(q.c + i) * K + a : (int64_t)K * p.D + q.c + i] = s;
            }
        }
    }
}

// the gradient of the K-1 rows before the first token: a thread per element
template <typename T> __global__ __launch_bounds__(NT) void merit_cconv_dinit(CconvParams p)
{
    const int K = p.K;
    const int64_t id = (int64_t)blockIdx.x * NT + threadIdx.x;
    if (id >= p.B * (K - 1) * p.D) return;
    const int64_t row = id / p.D, b = row / (K - 1);
    const int c = (int)(id - row * p.D), i = (int)(row - b * (K - 1));
    const int64_t n = p.lens ? min((int64_t)max(p.lens[b], 0), p.L) : p.L;
    const int64_t t = i - (K - 1);
    float g = 0.0f;
    for (int a = 0; a < K; ++a) {
        const int64_t s = t + K - 1 - a;
        if (s < 0 || s >= n) continue;
        float u = load_param<T>(p.b, c, 0.0f);
        for (int e = 0; e < K; ++e) {
            const int64_t r = s + e - (K - 1);
            float v = 0.0f;
            if (r >= 0) v = (float)static_cast<const T *>(p.x.data)[b * p.x.s0 + r * p.x.s1 + c];
            else if (p.init.data) v = (float)static_cast<const T *>(p.init.data)[b * p.init.s0 + (K - 1 + r) * p.init.s1 + c];
            u = fmaf(load_param<T>(p.w, (int64_t)c * K + e, 0.0f), v, u);
        }
        const float d = (float)static_cast<const T *>(p.dy.data)[b * p.dy.s0 + s * p.dy.s1 + c] * act_slope(u, p.act);
        g = fmaf(load_param<T>(p.w, (int64_t)c * K + a, 0.0f), d, g);
    }
    if (p.dfin.data && t >= n - (K - 1))
        g += (float)static_cast<const T *>(p.dfin.data)[b * p.dfin.s0 + (t - (n - (K - 1))) * p.dfin.s1 + c];
    static_cast<T *>(p.dinit.data)[b * p.dinit.s0 + i * p.dinit.s1 + c] = (T)g;
}

template <typename T, int V, int K> __global__ __launch_bounds__(NT) void merit_cconv_step(CconvParams p)
{
    const int cu = p.D / V;
    const int64_t id = (int64_t)blockIdx.x * NT + threadIdx.x;
    const int64_t s = id / cu;
    if (s >= p.B) return;
    const int c = (int)(id - s * cu) * V;
    float w[K][V], b[V];
    vec_t<T, V> row[K], o;
#pragma unroll
    for (int j = 0; j < K - 1; ++j) row[j] = load_vec<T, V>(p.init.data, s * p.init.s0 + j * p.init.s1 + c);
    row[K - 1] = load_vec<T, V>(p.x.data, s * p.x.s0 + c);
    load_taps<T, V, K>(p, c, w, b);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float u = b[i];
#pragma unroll
        for (int a = 0; a < K; ++a) u = fmaf(w[a][i], at<T, V>(row[a], i), u);
        put<T, V>(o, i, apply_act(u, p.act));
    }
    store_vec<T, V>(p.y.data, s * p.y.s0 + c, o);
#pragma unroll
    for (int j = 0; j < K - 1; ++j) store_vec<T, V>(p.fin.data, s * p.fin.s0 + j * p.fin.s1 + c, row[j + 1]);
}

// ---- launches -------------------------------------------------------------------------
enum { FORWARD, BACKWARD, STEP };

template <typename T, int V, int K> hipError_t launch_k(const CconvParams &p, int pass, hipStream_t s)
{
    const int cu = p.D / V;
    if (pass == STEP) {
        merit_cconv_step<T, V, K><<<(unsigned)((p.B * cu + NT - 1) / NT), NT, 0, s>>>(p);
        return hipGetLastError();
    }
    int ct = 1;
    while (ct < 64 && ct < cu) ct *= 2;
    const unsigned grid = (unsigned)(p.row_blocks * ((cu + ct - 1) / ct));
    if (pass == FORWARD) {
        merit_cconv<T, V, K><<<grid, NT, 0, s>>>(p);
        return hipGetLastError();
    }
    merit_cconv_backward<T, V, K><<<grid, NT, 0, s>>>(p);
    if (p.dinit.data && K > 1) {
        const int64_t count = p.B * (K - 1) * p.D;
        merit_cconv_dinit<T><<<(unsigned)((count + NT - 1) / NT), NT, 0, s>>>(p);
    }
    if (p.dw || p.db) {
        ReduceParams r = {};
        r.in = p.part;
        r.rows = p.row_blocks;
        r.pitch = (int64_t)(K + 1) * p.D;
        r.nseg = 2;
        r.seg[0] = {p.dw, 0, (int64_t)K * p.D};
        r.seg[1] = {p.db, (int64_t)K * p.D, p.D};
        return launch_reduce_rows(r, s);
    }
    return hipGetLastError();
}

template <typename T, int V> hipError_t launch_v(const CconvParams &p, int pass, hipStream_t s)
{
    switch (p.K) {
    case 1: return launch_k<T, V, 1>(p, pass, s);
    case 2: return launch_k<T, V, 2>(p, pass, s);
    case 3: return launch_k<T, V, 3>(p, pass, s);
    case 4: return launch_k<T, V, 4>(p, pass, s);
    case 5: return launch_k<T, V, 5>(p, pass, s);
    case 6: return launch_k<T, V, 6>(p, pass, s);
    case 7: return launch_k<T, V, 7>(p, pass, s);
    default: return launch_k<T, V, 8>(p, pass, s);
    }
}

hipError_t launch_type(const CconvParams &p, int type, int pass, hipStream_t s)
{
    if (type == MERIT_F32) return p.vec == 4 ? launch_v<float, 4>(p, pass, s) : launch_v<float, 1>(p, pass, s);
    if (type == MERIT_F16) return p.vec == 4 ? launch_v<f16_t, 4>(p, pass, s) : launch_v<f16_t, 1>(p, pass, s);
    return p.vec == 4 ? launch_v<bf16_t, 4>(p, pass, s) : launch_v<bf16_t, 1>(p, pass, s);
}

}  // namespace

hipError_t launch_cconv(const CconvParams &p, int type, hipStream_t s) { return launch_type(p, type, FORWARD, s); }
hipError_t launch_cconv_backward(const CconvParams &p, int type, hipStream_t s) { return launch_type(p, type, BACKWARD, s); }
hipError_t launch_cconv_step(const CconvParams &p, int type, hipStream_t s) { return launch_type(p, type, STEP, s); }

}  // namespace merit
