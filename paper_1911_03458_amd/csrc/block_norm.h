// The norms before and after a block with its gate and residual scale, rows of C channels:
//     u = norm(x) aw + ab,   t = u act(z),   out = r + s t,   n = norm(out) bw + bb
//     norm(x) = (x - mean) rstd, the mean 0 where it is not a layer norm
// and backward, with g = dn bw, oh = norm(out) (of the unrounded result, computed again from its row):
//     do = dout + rstd (g - [mean g] - oh mean(g oh)),   dr = do,   ds = sum do t,   dt = s do
//     dz = dt u act'(z),   du = dt act(z),   dx = rstd (du aw - [mean(du aw)] - xh mean(du aw xh)),   daw = sum du xh, dab = sum du, ..
// Bound by memory, rows of one head by their instructions as well (30 a value forward with a SiLU gate).  A row is held in
// registers by a run of lanes, or a workgroup of 256 or 512 threads, so every tensor is read once; a thread keeps its columns
// while it walks down the rows, which keeps parameters and the sums of their gradients in registers, and asks for the next row
// before it works on this one (backward, 16384 rows of 2048: 85 us against 139 without).  bf16, the bytes at their rate: 16384
// rows of 2048, both norms, forward 49 us (5.5 TB/s), with an fp32 stream 77 us (5.2), backward 85 us (4.7); 262144 rows of 128,
// after-norm and gate, forward 44 us (4.6), backward 68 us (5.0).
// Rows of more than 8 values a thread that are not in pieces of 16 bytes spill: 2048 of 8191, fp32, backward, 0.34 ms.
#pragma once

#include "merit_internal.h"
#include "tokens.h"

namespace merit {
namespace block_norm {

// V values of a row side by side, moved in pieces of at most 16 bytes (rows start on such pieces)
template <typename T, int V> struct Piece {
    static constexpr int bytes = V * (int)sizeof(T) < 16 ? V * (int)sizeof(T) : 16, count = V * (int)sizeof(T) / bytes;
    T v[V];
};
template <typename T, int V> __device__ __forceinline__ Piece<T, V> load_piece(const void *base, int64_t at)
{
    typedef Piece<T, V> P;
    typedef vec_t<T, P::bytes / (int)sizeof(T)> W;
    const T *from = static_cast<const T *>(base) + at;
    P r;
#pragma unroll
    for (int i = 0; i < P::count; ++i) {
        const W w = reinterpret_cast<const W *>(from)[i];
        __builtin_memcpy(r.v + i * (P::bytes / (int)sizeof(T)), &w, P::bytes);
    }
    return r;
}
template <typename T, int V> __device__ __forceinline__ void store_piece(void *base, int64_t at, const float (&f)[V])
{
    typedef Piece<T, V> P;
    constexpr int N = P::bytes / (int)sizeof(T);
    typedef vec_t<T, N> W;
    T *to = static_cast<T *>(base) + at;
#pragma unroll
    for (int i = 0; i < P::count; ++i) {
        W w;
#pragma unroll
        for (int e = 0; e < N; ++e) put<T, N>(w, e, f[i * N + e]);
        reinterpret_cast<W *>(to)[i] = w;
    }
}
template <typename T, int V> __device__ __forceinline__ Piece<T, V> no_piece()
{
    Piece<T, V> r;
#pragma unroll
    for (int e = 0; e < V; ++e) r.v[e] = (T)0.0f;
    return r;
}

// A form of the kernels: which norms there are, in bits, as root mean squares without biases; 0 reads all that from the
// arguments.  What a form leaves out takes no registers and no instructions: backward, bf16, 262144 rows of 128 with an
// after-norm and a gate 69 us against 113, 16384 rows of 2048 with both norms 85 against 103.
template <int FORM> struct Form {
    static __device__ __forceinline__ bool after(const BlockNormParams &p) { return FORM ? (FORM & 1) != 0 : p.after != 0; }
    static __device__ __forceinline__ bool before(const BlockNormParams &p) { return FORM ? (FORM & 2) != 0 : p.before != 0; }
    static __device__ __forceinline__ bool layer(const BlockNormParams &p) { return !FORM && p.layer; }
};

// act(z), and its slope.  The choice is the same for all values, so it is outside of their loop.
template <int V> __device__ __forceinline__ void gates(const float (&z)[V], int act, float (&v)[V])
{
    if (act == MERIT_ACT_SIGMOID) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = sigmoidf(z[e]);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = z[e];
        if (act == MERIT_ACT_SILU) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = apply_act(z[e], MERIT_ACT_SILU);
        } else if (act == MERIT_ACT_RELU) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = apply_act(z[e], MERIT_ACT_RELU);
        }
    }
}
template <int V> __device__ __forceinline__ void gate_slopes(const float (&z)[V], int act, float (&v)[V], float (&slope)[V])
{
    gates<V>(z, act, v);
    if (act == MERIT_ACT_SIGMOID) {
#pragma unroll
        for (int e = 0; e < V; ++e) slope[e] = v[e] * (1.0f - v[e]);
    } else if (act == MERIT_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < V; ++e) slope[e] = act_slope(z[e], MERIT_ACT_SILU);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) slope[e] = act == MERIT_ACT_RELU ? act_slope(z[e], MERIT_ACT_RELU) : 1.0f;
    }
}

// Where a thread's channels and rows are
struct Place {
    int first, step;       // vectors
    int64_t row0, rstep;   // rows of the workgroup, or of the wavefront
    int sub;               // the row of those that a wavefront takes at once
};
template <int NT> __device__ __forceinline__ Place place(const BlockNormParams &p)
{
    Place q;
    if (p.lanes) {
        const int each = 64 / p.lanes, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        q.first = lane & (p.lanes - 1);
        q.step = p.lanes;
        q.sub = lane / p.lanes;
        q.row0 = ((int64_t)blockIdx.x * (NT / 64) + wave) * each;
        q.rstep = (int64_t)gridDim.x * (NT / 64) * each;
    } else {
        q.first = threadIdx.x;
        q.step = NT;
        q.sub = 0;
        q.row0 = blockIdx.x;
        q.rstep = gridDim.x;
    }
    return q;
}

// The rows of a thread one by one, without divisions and products.  (Backward the places of eight tensors would take registers
// that the sums need: 262144 rows of 128, bf16, after-norm and gate, 94 against 68 us.)
struct Line {
    int64_t at, go, wrap;  // elements from the tensor's start; the way to the next row, and where it is in a later sequence
};
struct Walk {
    uint32_t b, t, sequences, step, L;
    __device__ __forceinline__ Walk(const BlockNormParams &p, const Place &q) : L((uint32_t)p.L)
    {
        b = (uint32_t)(q.row0 + q.sub) / L;
        t = (uint32_t)(q.row0 + q.sub) - b * L;
        sequences = (uint32_t)q.rstep / L;
        step = (uint32_t)q.rstep - sequences * L;
    }
    __device__ __forceinline__ Line line(const Rows &r) const
    {
        Line n = {b * r.s0 + t * r.s1, sequences * r.s0 + step * r.s1, 0};
        n.wrap = n.go + r.s0 - L * r.s1;
        return n;
    }
    template <int N> __device__ __forceinline__ void next(Line (&lines)[N])
    {
        t += step;
        const bool over = t >= L;
        if (over) t -= L;
#pragma unroll
        for (int i = 0; i < N; ++i) lines[i].at += over ? lines[i].wrap : lines[i].go;
    }
};

// Sums over a row's threads.  `turn` alternates between two halves of the LDS: a sum's values are read before the next one's
// barrier, and written over after it.
template <int NT, int N> __device__ __forceinline__ void sum_row(float (&v)[N], int lanes, float (*slots)[2][NT / 64], int &turn)
{
    if (lanes) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = sum_lanes(v[i], lanes);
        return;
    }
    turn ^= 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = sum_lanes(v[i], 64);
        if ((threadIdx.x & 63) == 0) slots[turn][i][threadIdx.x >> 6] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float s = slots[turn][i][0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) s += slots[turn][i][w];
        v[i] = s;
    }
}

// A parameter's values at a thread's channels, kept in registers or read again for each row; zeros where it has none, so
// that what it makes of the zeros that it holds for them adds nothing to a row's sums
template <typename T, int V, int U, bool HOLD> struct Vector {
    float v[HOLD ? U : 1][V];
    Param from;
    float absent;
    __device__ __forceinline__ Vector(Param p, float missing, const int (&c)[U], const bool (&has)[U]) : from(p), absent(missing)
    {
        if constexpr (HOLD)
#pragma unroll
            for (int j = 0; j < U; ++j) read(c[j], has[j], v[j]);
    }
    __device__ __forceinline__ void read(int c, bool has, float (&out)[V]) const
    {
        load_params<T>(from, c, absent, out);
#pragma unroll
        for (int e = 0; e < V; ++e) out[e] = has ? out[e] : 0.0f;
    }
    __device__ __forceinline__ void get(int j, int c, bool has, float (&out)[V]) const
    {
        if constexpr (HOLD)
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = v[j][e];
        else read(c, has, out);
    }
};

// norm(f) in place, zeros where a thread has no channels; the mean (0 without `layer`) and 1 / root
template <int NT, int V, int U, int FORM>
__device__ __forceinline__ void normalise(float (&f)[U][V], const bool (&ok)[U], const BlockNormParams &p, float (*slots)[2][NT / 64],
                                          int &turn, float &mean, float &rstd)
{
    const float inv = 1.0f / (float)p.C;
    mean = 0.0f;
    if (Form<FORM>::layer(p)) {
        float s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += f[j][e];
        sum_row<NT, 1>(s, p.lanes, slots, turn);
        mean = s[0] * inv;
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (Form<FORM>::layer(p)) f[j][e] = ok[j] ? f[j][e] - mean : 0.0f;
            s[0] = fmaf(f[j][e], f[j][e], s[0]);
        }
    sum_row<NT, 1>(s, p.lanes, slots, turn);
    rstd = __builtin_amdgcn_rsqf(s[0] * inv + p.eps);
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) f[j][e] *= rstd;
}

template <typename T, typename R, int V, int U, int NT, int FORM>
__global__ __launch_bounds__(NT) void merit_block_norm_rows(BlockNormParams p)
{
    __shared__ float slots[2][2][NT / 64];
    typedef Form<FORM> F;
    int turn = 0;
    const Place q = place<NT>(p);
    bool has[U];
    int c[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const int u = q.first + j * q.step;
        has[j] = u * V < p.C;
        c[j] = has[j] ? u * V : 0;
    }
    const Vector<T, V, U, true> aw(p.aw, 1.0f, c, has), ab(FORM ? Param{} : p.ab, 0.0f, c, has), sc(p.scale, 1.0f, c, has);
    const Vector<T, V, U, true> bw(p.bw, 1.0f, c, has), bb(FORM ? Param{} : p.bb, 0.0f, c, has);
    Piece<T, V> xn[U], zn[U];
    Piece<R, V> rn[U];
    Walk in(p, q), to(p, q);
    Line from[3] = {in.line(p.x), in.line(p.z), in.line(p.r)};
    Line out[2] = {to.line(p.out), to.line(p.n)};
#pragma unroll
    for (int j = 0; j < U; ++j) {
        xn[j] = no_piece<T, V>();
        zn[j] = no_piece<T, V>();
        rn[j] = no_piece<R, V>();
    }
    auto load = [&](int64_t r0) __attribute__((always_inline)) {
        if (r0 + q.sub < p.rows)
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (!has[j]) continue;
                xn[j] = load_piece<T, V>(p.x.data, from[0].at + c[j]);
                if (p.z.data) zn[j] = load_piece<T, V>(p.z.data, from[1].at + c[j]);
                if (p.r.data) rn[j] = load_piece<R, V>(p.r.data, from[2].at + c[j]);
            }
        in.next(from);
    };
    if (q.row0 < p.rows) load(q.row0);
    for (int64_t r0 = q.row0; r0 < p.rows; r0 += q.rstep) {
        const int64_t row = r0 + q.sub;
        const bool live = row < p.rows;
        float f[U][V], z[U][V], r[U][V];
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                f[j][e] = (float)xn[j].v[e];
                z[j][e] = (float)zn[j].v[e];
                r[j][e] = (float)rn[j].v[e];
            }
        if (r0 + q.rstep < p.rows) load(r0 + q.rstep);
        float mean, rstd;
        if (F::after(p)) {
            normalise<NT, V, U, FORM>(f, has, p, slots, turn, mean, rstd);
            if (live && q.first == 0) {
                if (p.am) p.am[row] = mean;
                if (p.ar) p.ar[row] = rstd;
            }
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            float w[V], bias[V], s[V];
            aw.get(j, c[j], has[j], w);
            ab.get(j, c[j], has[j], bias);
            sc.get(j, c[j], has[j], s);
            if (p.z.data) gates<V>(z[j], p.act, z[j]);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float u = F::after(p) ? fmaf(f[j][e], w[e], bias[e]) : f[j][e];
                if (p.z.data) u *= z[j][e];
                f[j][e] = fmaf(s[e], u, r[j][e]);
            }
        }
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (live && has[j]) store_piece<R, V>(p.out.data, out[0].at + c[j], f[j]);
        if (F::before(p)) {
            normalise<NT, V, U, FORM>(f, has, p, slots, turn, mean, rstd);
            if (live && q.first == 0) {
                if (p.bm) p.bm[row] = mean;
                if (p.br) p.br[row] = rstd;
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float o[V], w[V], bias[V];
                bw.get(j, c[j], has[j], w);
                bb.get(j, c[j], has[j], bias);
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] = fmaf(f[j][e], w[e], bias[e]);
                if (live && has[j]) store_piece<T, V>(p.n.data, out[1].at + c[j], o);
            }
        }
        to.next(out);
    }
}

template <typename T, typename R, int V, int U, int NT, int FORM>
__global__ __launch_bounds__(NT, FORM == 1 && V * U <= 8 ? 4 : 1) void merit_block_norm_rows_backward(BlockNormParams p)
{
    __shared__ float slots[2][2][NT / 64];
    __shared__ float red[NT == 256 ? NT : 1][V];
    typedef Form<FORM> F;
    int turn = 0;
    const Place q = place<NT>(p);
    const float inv = 1.0f / (float)p.C;
    float sums[5][U][V];
    bool has[U];
    int c[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const int u = q.first + j * q.step;
        has[j] = u * V < p.C;
        c[j] = has[j] ? u * V : 0;
#pragma unroll
        for (int k = 0; k < 5; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) sums[k][j][e] = 0.0f;
    }
    // 16 values a thread leave no registers for parameters and the next row (4096 rows of 8192, bf16,
    // both norms: 122 us; 1024 threads of 8 values, all of them in 128 registers each, took 594)
    constexpr bool HOLD = V * U < 16, AHEAD = HOLD;
    const Vector<T, V, U, HOLD> aw(p.aw, 1.0f, c, has), ab(FORM ? Param{} : p.ab, 0.0f, c, has), sc(p.scale, 1.0f, c, has), bw(p.bw, 1.0f, c, has);
    Piece<T, V> xn[U], zn[U], nn[U];
    Piece<R, V> rn[U], dn[U];
    float an[2], bn[2];
    auto load = [&](int64_t r0) __attribute__((always_inline)) {
        const int64_t row = r0 + q.sub;
        const bool live = row < p.rows;
        const uint32_t b = (uint32_t)row / (uint32_t)p.L, t = (uint32_t)row - b * (uint32_t)p.L;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            xn[j] = no_piece<T, V>();
            zn[j] = no_piece<T, V>();
            nn[j] = no_piece<T, V>();
            rn[j] = no_piece<R, V>();
            dn[j] = no_piece<R, V>();
            if (!live || !has[j]) continue;
            xn[j] = load_piece<T, V>(p.x.data, b * p.x.s0 + t * p.x.s1 + c[j]);
            if (p.z.data) zn[j] = load_piece<T, V>(p.z.data, b * p.z.s0 + t * p.z.s1 + c[j]);
            if (F::before(p)) {
                nn[j] = load_piece<T, V>(p.dn.data, b * p.dn.s0 + t * p.dn.s1 + c[j]);
                if (p.r.data) rn[j] = load_piece<R, V>(p.r.data, b * p.r.s0 + t * p.r.s1 + c[j]);
            }
            if (p.dout.data) dn[j] = load_piece<R, V>(p.dout.data, b * p.dout.s0 + t * p.dout.s1 + c[j]);
        }
        an[0] = live && F::after(p) && F::layer(p) ? p.am[row] : 0.0f;
        an[1] = live && F::after(p) ? p.ar[row] : 0.0f;
        bn[0] = live && F::before(p) && F::layer(p) ? p.bm[row] : 0.0f;
        bn[1] = live && F::before(p) ? p.br[row] : 0.0f;
    };
    if (AHEAD && q.row0 < p.rows) load(q.row0);
    for (int64_t r0 = q.row0; r0 < p.rows; r0 += q.rstep) {
        const int64_t row = r0 + q.sub;
        const bool live = row < p.rows;
        const uint32_t b = (uint32_t)row / (uint32_t)p.L, t = (uint32_t)row - b * (uint32_t)p.L;
        if (!AHEAD) load(r0);
        const float am = an[0], ar = an[1], bm = bn[0], br = bn[1];
        float d[U][V], xh[U][V], u[U][V], act[U][V], slope[U][V], r[U][V], g[U][V];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            float z[V], w[V], bias[V];
            aw.get(j, c[j], true, w);
            ab.get(j, c[j], true, bias);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float x = (float)xn[j].v[e];
                z[e] = (float)zn[j].v[e];
                r[j][e] = (float)rn[j].v[e];
                g[j][e] = (float)nn[j].v[e];
                d[j][e] = (float)dn[j].v[e];
                xh[j][e] = F::after(p) ? (x - am) * ar : x;
                u[j][e] = F::after(p) ? fmaf(xh[j][e], w[e], bias[e]) : x;
                act[j][e] = 1.0f;
                slope[j][e] = 0.0f;
            }
            if (p.z.data) gate_slopes<V>(z, p.act, act[j], slope[j]);
        }
        if (AHEAD && r0 + q.rstep < p.rows) load(r0 + q.rstep);
        if (F::before(p)) {
            float s[2] = {0.0f, 0.0f}, oh[U][V];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float w[V], scale[V];
                bw.get(j, c[j], true, w);
                sc.get(j, c[j], true, scale);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float o = fmaf(scale[e], u[j][e] * act[j][e], r[j][e]);
                    oh[j][e] = live && has[j] ? (o - bm) * br : 0.0f;
                    sums[3][j][e] = fmaf(g[j][e], oh[j][e], sums[3][j][e]);
                    if (!FORM) sums[4][j][e] += g[j][e];
                    g[j][e] *= w[e];
                    s[0] += g[j][e];
                    s[1] = fmaf(g[j][e], oh[j][e], s[1]);
                }
            }
            float m1 = 0.0f, m2;
            if (F::layer(p)) {
                sum_row<NT, 2>(s, p.lanes, slots, turn);
                m1 = s[0] * inv;
                m2 = s[1] * inv;
            } else {
                float one[1] = {s[1]};
                sum_row<NT, 1>(one, p.lanes, slots, turn);
                m2 = one[0] * inv;
            }
#pragma unroll
            for (int j = 0; j < U; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) d[j][e] = fmaf(br, g[j][e] - m1 - oh[j][e] * m2, d[j][e]);
        }
        if (p.dr.data)
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (live && has[j]) store_piece<R, V>(p.dr.data, b * p.dr.s0 + t * p.dr.s1 + c[j], d[j]);
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (!(live && has[j])) continue;
            float dz[V], w[V], scale[V];
            aw.get(j, c[j], true, w);
            sc.get(j, c[j], true, scale);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float dt = d[j][e] * scale[e], du = dt * act[j][e];
                sums[2][j][e] = fmaf(d[j][e], u[j][e] * act[j][e], sums[2][j][e]);
                dz[e] = dt * u[j][e] * slope[j][e];
                sums[0][j][e] = fmaf(du, xh[j][e], sums[0][j][e]);
                if (!FORM) sums[1][j][e] += du;
                d[j][e] = F::after(p) ? du * w[e] : du;
                s[0] += d[j][e];
                s[1] = fmaf(d[j][e], xh[j][e], s[1]);
            }
            if (p.dz.data) store_piece<T, V>(p.dz.data, b * p.dz.s0 + t * p.dz.s1 + c[j], dz);
        }
        if (F::after(p)) {
            float m1 = 0.0f, m2;
            if (F::layer(p)) {
                sum_row<NT, 2>(s, p.lanes, slots, turn);
                m1 = s[0] * inv;
                m2 = s[1] * inv;
            } else {
                float one[1] = {s[1]};
                sum_row<NT, 1>(one, p.lanes, slots, turn);
                m2 = one[0] * inv;
            }
#pragma unroll
            for (int j = 0; j < U; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) d[j][e] = ar * (d[j][e] - m1 - xh[j][e] * m2);
        }
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (live && has[j]) store_piece<T, V>(p.dx.data, b * p.dx.s0 + t * p.dx.s1 + c[j], d[j]);
    }
    const float *want[5] = {p.daw, p.dab, p.dscale, p.dbw, p.dbb};
    float *part = p.part + (int64_t)blockIdx.x * 5 * p.C;
#pragma unroll
    for (int k = 0; k < 5; ++k) {
        if (!want[k]) continue;
        if (NT == 256 && p.lanes) {         // threads with the same columns
            __syncthreads();
#pragma unroll
            for (int e = 0; e < V; ++e) red[threadIdx.x % (NT == 256 ? NT : 1)][e] = sums[k][0][e];
            __syncthreads();
            if ((int)threadIdx.x < p.lanes && has[0])
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float v = 0.0f;
                    for (int i = threadIdx.x; i < NT; i += p.lanes) v += red[i % (NT == 256 ? NT : 1)][e];
                    part[k * p.C + c[0] + e] = v;
                }
        } else {
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (has[j])
#pragma unroll
                    for (int e = 0; e < V; ++e) part[k * p.C + c[j] + e] = sums[k][j][e];
        }
    }
}

template <bool BACKWARD, typename T, typename R, int V, int U, int NT, int FORM> hipError_t launch_form(const BlockNormParams &p, hipStream_t s)
{
    if constexpr (BACKWARD) merit_block_norm_rows_backward<T, R, V, U, NT, FORM><<<(unsigned)p.blocks, NT, 0, s>>>(p);
    else merit_block_norm_rows<T, R, V, U, NT, FORM><<<(unsigned)p.blocks, NT, 0, s>>>(p);
    return hipGetLastError();
}
template <bool BACKWARD, typename T, typename R, int V, int U, int NT> hipError_t launch_rows(const BlockNormParams &p, hipStream_t s)
{
    // (pieces of 16 bytes and the longest rows: the others wait on the number of their loads)
    if constexpr (V * sizeof(T) == 16 || V * U == 16) {
        if (!p.layer && !p.ab.data && !p.bb.data && !p.dab && !p.dbb) {
            if (p.after && p.before) return launch_form<BACKWARD, T, R, V, U, NT, 3>(p, s);
            return p.after ? launch_form<BACKWARD, T, R, V, U, NT, 1>(p, s) : launch_form<BACKWARD, T, R, V, U, NT, 2>(p, s);
        }
    }
    return launch_form<BACKWARD, T, R, V, U, NT, 0>(p, s);
}
template <bool BACKWARD, typename T, typename R, int V> hipError_t launch_vec(const BlockNormParams &p, hipStream_t s)
{
    if (p.threads == 256) return launch_rows<BACKWARD, T, R, V, 1, 256>(p, s);
    // (rows of at most MERIT_BLOCK_NORM_MAX_CHANNELS: 16 values a thread)
    if (p.units == 1) return launch_rows<BACKWARD, T, R, V, 1, 512>(p, s);
    if (p.units == 2) return launch_rows<BACKWARD, T, R, V, 2, 512>(p, s);
    if constexpr (V <= 4) if (p.units == 4) return launch_rows<BACKWARD, T, R, V, 4, 512>(p, s);
    if constexpr (V <= 2) if (p.units == 8) return launch_rows<BACKWARD, T, R, V, 8, 512>(p, s);
    if constexpr (V <= 1) if (p.units == 16) return launch_rows<BACKWARD, T, R, V, 16, 512>(p, s);
    return hipErrorInvalidValue;
}
template <bool BACKWARD, typename T, typename R> hipError_t launch_typed(const BlockNormParams &p, hipStream_t s)
{
    if constexpr (sizeof(T) == 2) {
        if (p.vec == 8) return launch_vec<BACKWARD, T, R, 8>(p, s);
    } else {
        if (p.vec == 4) return launch_vec<BACKWARD, T, R, 4>(p, s);
    }
    return p.vec == 2 ? launch_vec<BACKWARD, T, R, 2>(p, s) : launch_vec<BACKWARD, T, R, 1>(p, s);
}
// The passes of one type, each in a file of its own (block_norm_*.hip)
template <typename T> hipError_t passes(const BlockNormParams &p, bool backward, hipStream_t s)
{
    if constexpr (sizeof(T) == 4) return backward ? launch_typed<true, T, float>(p, s) : launch_typed<false, T, float>(p, s);
    else if (p.stream == MERIT_F32) return backward ? launch_typed<true, T, float>(p, s) : launch_typed<false, T, float>(p, s);
    else return backward ? launch_typed<true, T, T>(p, s) : launch_typed<false, T, T>(p, s);
}
hipError_t passes_f32(const BlockNormParams &p, bool backward, hipStream_t s);
hipError_t passes_f16(const BlockNormParams &p, bool backward, hipStream_t s);
hipError_t passes_bf16(const BlockNormParams &p, bool backward, hipStream_t s);

}  // namespace block_norm
}  // namespace merit
