// The norms before and after a block with its gate and residual scale, rows of C channels:
//     u = norm(x) aw + ab,   t = u act(z),   out = r + s t,   n = norm(out) bw + bb
//     norm(x) = (x - mean) rstd, the mean 0 where it is not a layer norm
// and backward, with g = dn bw, oh = norm(out) (of the unrounded result, computed again from its row):
//     do = dout + rstd (g - [mean g] - oh mean(g oh)),   dr = do,   ds = sum do t,   dt = s do
//     dz = dt u act'(z),   du = dt act(z),   dx = rstd (du aw - [mean(du aw)] - xh mean(du aw xh)),   daw = sum du xh, dab = sum du, ..
// Bound by memory.  A row is held in registers by a run of lanes, or a workgroup of 256 to 1024 threads, so every tensor is
// read once; a thread keeps its columns while it walks down the rows, which keeps parameters and the sums of their gradients
// in registers.
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

__device__ __forceinline__ float gate(float z, int act) { return act == MERIT_ACT_SIGMOID ? sigmoidf(z) : apply_act(z, act); }
__device__ __forceinline__ float gate_slope(float z, int act)
{
    if (act == MERIT_ACT_SIGMOID) {
        const float q = sigmoidf(z);
        return q * (1.0f - q);
    }
    return act_slope(z, act);
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

// norm(f) in place, absent values left out; the mean (0 without `layer`) and 1 / root
template <int NT, int V, int U>
__device__ __forceinline__ void normalise(float (&f)[U][V], const bool (&ok)[U], const BlockNormParams &p, float (*slots)[2][NT / 64],
                                          int &turn, float &mean, float &rstd)
{
    const float inv = 1.0f / (float)p.C;
    mean = 0.0f;
    if (p.layer) {
        float s[1] = {0.0f};
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += ok[j] ? f[j][e] : 0.0f;
        sum_row<NT, 1>(s, p.lanes, slots, turn);
        mean = s[0] * inv;
    }
    float s[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            f[j][e] = ok[j] ? f[j][e] - mean : 0.0f;
            s[0] = fmaf(f[j][e], f[j][e], s[0]);
        }
    sum_row<NT, 1>(s, p.lanes, slots, turn);
    rstd = __builtin_amdgcn_rsqf(s[0] * inv + p.eps);
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) f[j][e] *= rstd;
}

template <typename T, typename R, int V, int U, int NT>
__global__ __launch_bounds__(NT) void merit_block_norm_rows(BlockNormParams p)
{
    __shared__ float slots[2][2][NT / 64];
    int turn = 0;
    const Place q = place<NT>(p);
    float aw[U][V], ab[U][V], sc[U][V], bw[U][V], bb[U][V];
    bool has[U];
    int c[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const int u = q.first + j * q.step;
        has[j] = u * V < p.C;
        c[j] = has[j] ? u * V : 0;
        load_params<T>(p.aw, c[j], 1.0f, aw[j]);
        load_params<T>(p.ab, c[j], 0.0f, ab[j]);
        load_params<T>(p.scale, c[j], 1.0f, sc[j]);
        load_params<T>(p.bw, c[j], 1.0f, bw[j]);
        load_params<T>(p.bb, c[j], 0.0f, bb[j]);
    }
    Piece<T, V> xn[U], zn[U];
    Piece<R, V> rn[U];
    auto load = [&](int64_t r0) __attribute__((always_inline)) {
        const int64_t r = r0 + q.sub;
        const bool live = r < p.rows;
        const uint32_t b = (uint32_t)r / (uint32_t)p.L, t = (uint32_t)r - b * (uint32_t)p.L;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            xn[j] = no_piece<T, V>();
            zn[j] = no_piece<T, V>();
            rn[j] = no_piece<R, V>();
            if (!live || !has[j]) continue;
            xn[j] = load_piece<T, V>(p.x.data, b * p.x.s0 + t * p.x.s1 + c[j]);
            if (p.z.data) zn[j] = load_piece<T, V>(p.z.data, b * p.z.s0 + t * p.z.s1 + c[j]);
            if (p.r.data) rn[j] = load_piece<R, V>(p.r.data, b * p.r.s0 + t * p.r.s1 + c[j]);
        }
    };
    if (q.row0 < p.rows) load(q.row0);
    for (int64_t r0 = q.row0; r0 < p.rows; r0 += q.rstep) {
        const int64_t row = r0 + q.sub;
        const bool live = row < p.rows;
        const uint32_t b = (uint32_t)row / (uint32_t)p.L, t = (uint32_t)row - b * (uint32_t)p.L;
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
        if (p.after) {
            normalise<NT, V, U>(f, has, p, slots, turn, mean, rstd);
            if (live && q.first == 0) {
                if (p.am) p.am[row] = mean;
                if (p.ar) p.ar[row] = rstd;
            }
        }
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float u = p.after ? fmaf(f[j][e], aw[j][e], ab[j][e]) : f[j][e];
                if (p.z.data) u *= gate(z[j][e], p.act);
                f[j][e] = fmaf(sc[j][e], u, r[j][e]);
            }
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (live && has[j]) store_piece<R, V>(p.out.data, b * p.out.s0 + t * p.out.s1 + c[j], f[j]);
        if (p.before) {
            normalise<NT, V, U>(f, has, p, slots, turn, mean, rstd);
            if (live && q.first == 0) {
                if (p.bm) p.bm[row] = mean;
                if (p.br) p.br[row] = rstd;
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float o[V];
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] = fmaf(f[j][e], bw[j][e], bb[j][e]);
                if (live && has[j]) store_piece<T, V>(p.n.data, b * p.n.s0 + t * p.n.s1 + c[j], o);
            }
        }
    }
}

template <typename T, typename R, int V, int U, int NT>
__global__ __launch_bounds__(NT) void merit_block_norm_rows_backward(BlockNormParams p)
{
    __shared__ float slots[2][2][NT / 64];
    __shared__ float red[NT == 256 ? NT : 1][V];
    int turn = 0;
    const Place q = place<NT>(p);
    const float inv = 1.0f / (float)p.C;
    float aw[U][V], ab[U][V], sc[U][V], bw[U][V], sums[5][U][V];
    bool has[U];
    int c[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const int u = q.first + j * q.step;
        has[j] = u * V < p.C;
        c[j] = has[j] ? u * V : 0;
        load_params<T>(p.aw, c[j], 1.0f, aw[j]);
        load_params<T>(p.ab, c[j], 0.0f, ab[j]);
        load_params<T>(p.scale, c[j], 1.0f, sc[j]);
        load_params<T>(p.bw, c[j], 1.0f, bw[j]);
#pragma unroll
        for (int k = 0; k < 5; ++k)
#pragma unroll
            for (int e = 0; e < V; ++e) sums[k][j][e] = 0.0f;
    }
    for (int64_t r0 = q.row0; r0 < p.rows; r0 += q.rstep) {
        const int64_t row = r0 + q.sub;
        const bool live = row < p.rows;
        const uint32_t b = (uint32_t)row / (uint32_t)p.L, t = (uint32_t)row - b * (uint32_t)p.L;
        Piece<T, V> xv[U], zv[U], nv[U];
        Piece<R, V> rv[U], dv[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            xv[j] = no_piece<T, V>();
            zv[j] = no_piece<T, V>();
            nv[j] = no_piece<T, V>();
            rv[j] = no_piece<R, V>();
            dv[j] = no_piece<R, V>();
            if (!live || !has[j]) continue;
            xv[j] = load_piece<T, V>(p.x.data, b * p.x.s0 + t * p.x.s1 + c[j]);
            if (p.before) {
                nv[j] = load_piece<T, V>(p.dn.data, b * p.dn.s0 + t * p.dn.s1 + c[j]);
                if (p.r.data) rv[j] = load_piece<R, V>(p.r.data, b * p.r.s0 + t * p.r.s1 + c[j]);
            }
            if (p.dout.data) dv[j] = load_piece<R, V>(p.dout.data, b * p.dout.s0 + t * p.dout.s1 + c[j]);
            if (p.z.data) zv[j] = load_piece<T, V>(p.z.data, b * p.z.s0 + t * p.z.s1 + c[j]);
        }
        const float am = live && p.after && p.layer ? p.am[row] : 0.0f, ar = live && p.after ? p.ar[row] : 0.0f;
        const float bm = live && p.before && p.layer ? p.bm[row] : 0.0f, br = live && p.before ? p.br[row] : 0.0f;
        float d[U][V], xh[U][V], u[U][V], act[U][V];
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float x = (float)xv[j].v[e];
                d[j][e] = (float)dv[j].v[e];
                xh[j][e] = p.after ? (x - am) * ar : x;
                u[j][e] = p.after ? fmaf(xh[j][e], aw[j][e], ab[j][e]) : x;
                act[j][e] = p.z.data ? gate((float)zv[j].v[e], p.act) : 1.0f;
            }
        if (p.before) {
            float s[2] = {0.0f, 0.0f}, oh[U][V], g[U][V];
#pragma unroll
            for (int j = 0; j < U; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float dn = (float)nv[j].v[e], o = fmaf(sc[j][e], u[j][e] * act[j][e], (float)rv[j].v[e]);
                    oh[j][e] = live && has[j] ? (o - bm) * br : 0.0f;
                    sums[3][j][e] = fmaf(dn, oh[j][e], sums[3][j][e]);
                    sums[4][j][e] += dn;
                    g[j][e] = dn * bw[j][e];
                    s[0] += g[j][e];
                    s[1] = fmaf(g[j][e], oh[j][e], s[1]);
                }
            sum_row<NT, 2>(s, p.lanes, slots, turn);
            const float m1 = p.layer ? s[0] * inv : 0.0f, m2 = s[1] * inv;
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
            float dz[V];
            const bool in = live && has[j];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float dj = in ? d[j][e] : 0.0f, h = in ? xh[j][e] : 0.0f;
                sums[2][j][e] += in ? dj * (u[j][e] * act[j][e]) : 0.0f;
                const float dt = dj * sc[j][e], du = dt * act[j][e];
                dz[e] = p.z.data ? dt * u[j][e] * gate_slope((float)zv[j].v[e], p.act) : 0.0f;
                sums[0][j][e] += in ? du * h : 0.0f;
                sums[1][j][e] += in ? du : 0.0f;
                d[j][e] = p.after ? du * aw[j][e] : du;
                xh[j][e] = h;
                s[0] += in ? d[j][e] : 0.0f;
                s[1] += in ? d[j][e] * h : 0.0f;
            }
            if (p.dz.data && in) store_piece<T, V>(p.dz.data, b * p.dz.s0 + t * p.dz.s1 + c[j], dz);
        }
        if (p.after) {
            sum_row<NT, 2>(s, p.lanes, slots, turn);
            const float m1 = p.layer ? s[0] * inv : 0.0f, m2 = s[1] * inv;
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
    float *out = p.part + (int64_t)blockIdx.x * 5 * p.C;
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
                    out[k * p.C + c[0] + e] = v;
                }
        } else {
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (has[j])
#pragma unroll
                    for (int e = 0; e < V; ++e) out[k * p.C + c[j] + e] = sums[k][j][e];
        }
    }
}

template <bool BACKWARD, typename T, typename R, int V, int U, int NT> hipError_t launch_rows(const BlockNormParams &p, hipStream_t s)
{
    if constexpr (BACKWARD) merit_block_norm_rows_backward<T, R, V, U, NT><<<(unsigned)p.blocks, NT, 0, s>>>(p);
    else merit_block_norm_rows<T, R, V, U, NT><<<(unsigned)p.blocks, NT, 0, s>>>(p);
    return hipGetLastError();
}
template <bool BACKWARD, typename T, typename R, int V> hipError_t launch_vec(const BlockNormParams &p, hipStream_t s)
{
    if (p.threads == 256) return launch_rows<BACKWARD, T, R, V, 1, 256>(p, s);
    if (p.threads == 512) return launch_rows<BACKWARD, T, R, V, 1, 512>(p, s);
    // (rows of at most MERIT_BLOCK_NORM_MAX_CHANNELS: 16 values a thread)
    if (p.units == 1) return launch_rows<BACKWARD, T, R, V, 1, 1024>(p, s);
    if constexpr (V <= 8) if (p.units == 2) return launch_rows<BACKWARD, T, R, V, 2, 1024>(p, s);
    if constexpr (V <= 4) if (p.units == 4) return launch_rows<BACKWARD, T, R, V, 4, 1024>(p, s);
    if constexpr (V <= 2) if (p.units == 8) return launch_rows<BACKWARD, T, R, V, 8, 1024>(p, s);
    if constexpr (V <= 1) if (p.units == 16) return launch_rows<BACKWARD, T, R, V, 16, 1024>(p, s);
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
