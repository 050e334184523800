// Group norm with an activation, channels last, forward and backward:
//     y = act((x - mean) rstd w + b)      mean, var over the S positions x Cg channels of a group
//     du = dy act'(u),  g = du w,  xh = (x - mean) rstd
//     dx = rstd (g - mean(g) - xh mean(g xh)),   dw = sum du xh,   db = sum du
// Bound by memory: 2 (forward) or 3 (backward) passes of the tensor over HBM where it is read once.
//
// Three forms.  Measured (SiLU; a large copy reaches 6.0 TB/s):
//  - one row a group (S = 1, a token's heads): a group is a run of channels of one row.  A run of lanes, a wavefront or a
//    workgroup holds it in registers, so x is read once.  A wavefront keeps its columns and walks down the rows, which
//    keeps weights and the parameter gradients' sums in registers.  bfloat16, 16384 x 16 groups of 128 channels: 29 us
//    (4.7 TB/s); backward 41 us (4.9 TB/s) and 5 us of sums.  16 x 16 groups of 64: 3.5 us, a launch.
//  - a group a workgroup (the values of an image's group fit its registers): x is read once too.  bfloat16, 8x3136x256 in 32
//    groups 14.1 us (1.8 TB/s: 256 workgroups, so that every one loads, reduces and stores at the same time as all others).
//  - chunks (any S): workgroups reduce row chunks to partial statistics, a second launch joins them and applies; its read of x
//    comes from the cache behind the L2 where that holds the tensor.  binary16, 16x12544x64 in 8 groups (26 MB): 9.1 + 12.5 us
//    (3.6 TB/s, reads of both launches and the result); backward 15.6 + 16.2 us (4.0 TB/s) and 5 us of sums.
// Variances are sums of squared distances from a mean that is known by then (of the row, or of the batch of values in
// registers, batches joined by their counts): a mean far from zero costs no digits.
#include "merit_internal.h"
#include "tokens.h"

namespace merit {

namespace {

constexpr int NT = 256;

// ---------------------------------------------------------------------------
// one row a group
// ---------------------------------------------------------------------------
// Where a thread's channels are: unit j of U begins at channel c0 + j * step * V
struct RowPlace {
    int group, first, step, cu;
    bool active;
    int64_t row0, rstep;
};
__device__ __forceinline__ RowPlace row_place(int G, int cu, int lg, int wpg)
{
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    RowPlace q;
    q.cu = cu;
    if (wpg == 1) {
        q.group = (int)blockIdx.x * (64 / lg) + lane / lg;
        q.first = lane & (lg - 1);
        q.step = lg;
        q.row0 = (int64_t)blockIdx.y * 4 + wave;
        q.rstep = (int64_t)gridDim.y * 4;
    } else {
        q.group = (int)blockIdx.x;
        q.first = tid;
        q.step = NT;
        q.row0 = blockIdx.y;
        q.rstep = gridDim.y;
    }
    q.active = q.group < G;
    return q;
}

// the sum over a group's lanes; `slot`: four floats of LDS, not those of the sum before it
__device__ __forceinline__ float sum_group(float v, int lg, int wpg, float *slot)
{
    v = sum_lanes(v, lg);
    if (wpg == 1) return v;
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    return (slot[0] + slot[1]) + (slot[2] + slot[3]);
}

template <typename T, int V, int U>
__global__ __launch_bounds__(NT) void merit_norm_rows(NormParams p, int cu, int lg, int wpg)
{
    __shared__ float slots[2][4];
    const RowPlace q = row_place(p.G, cu, lg, wpg);
    const float inv = 1.0f / (float)p.Cg;
    float w[U][V], b[U][V];
    bool ok[U];
    int c[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const int u = q.first + j * q.step;
        ok[j] = q.active && u < q.cu;
        c[j] = q.group * p.Cg + u * V;
        load_params<T>(p.w, ok[j] ? c[j] : 0, 1.0f, w[j]);       // (a lane without channels: any, not used)
        load_params<T>(p.b, ok[j] ? c[j] : 0, 0.0f, b[j]);
    }
    vec_t<T, V> next[U] = {};
    if (q.row0 < p.N) {
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (ok[j]) next[j] = load_vec<T, V>(p.x.data, q.row0 * p.x.s0 + c[j]);
    }
    for (int64_t r = q.row0; r < p.N; r += q.rstep) {
        vec_t<T, V> now[U];
#pragma unroll
        for (int j = 0; j < U; ++j) now[j] = next[j];
        if (r + q.rstep < p.N) {
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (ok[j]) next[j] = load_vec<T, V>(p.x.data, (r + q.rstep) * p.x.s0 + c[j]);
        }
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) s += ok[j] ? at<T, V>(now[j], i) : 0.0f;
        const float mean = sum_group(s, lg, wpg, slots[0]) * inv;
        float m2 = 0.0f;
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = ok[j] ? at<T, V>(now[j], i) - mean : 0.0f;
                m2 = fmaf(d, d, m2);
            }
        const float rstd = __builtin_amdgcn_rsqf(sum_group(m2, lg, wpg, slots[1]) * inv + p.eps);
        if (q.active && q.first == 0) {
            if (p.mean) p.mean[r * p.G + q.group] = mean;
            if (p.rstd) p.rstd[r * p.G + q.group] = rstd;
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (!ok[j]) continue;
            vec_t<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i)
                put<T, V>(o, i, apply_act(fmaf((at<T, V>(now[j], i) - mean) * rstd, w[j][i], b[j][i]), p.act));
            store_vec<T, V>(p.y.data, r * p.y.s0 + c[j], o);
        }
    }
}

template <typename T, int V, int U>
__global__ __launch_bounds__(NT) void merit_norm_rows_backward(NormParams p, int cu, int lg, int wpg)
{
    __shared__ float slots[2][2][4];
    __shared__ float red[4][64][V];
    const RowPlace q = row_place(p.G, cu, lg, wpg);
    const float inv = 1.0f / (float)p.Cg;
    float w[U][V], b[U][V], s1[U][V], s2[U][V];
    bool ok[U];
    int c[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
        const int u = q.first + j * q.step;
        ok[j] = q.active && u < q.cu;
        c[j] = q.group * p.Cg + u * V;
        load_params<T>(p.w, ok[j] ? c[j] : 0, 1.0f, w[j]);
        load_params<T>(p.b, ok[j] ? c[j] : 0, 0.0f, b[j]);
#pragma unroll
        for (int i = 0; i < V; ++i) s1[j][i] = s2[j][i] = 0.0f;
    }
    for (int64_t r = q.row0; r < p.N; r += q.rstep) {
        const float mean = q.active ? p.mean[r * p.G + q.group] : 0.0f;
        const float rstd = q.active ? p.rstd[r * p.G + q.group] : 0.0f;
        vec_t<T, V> xv[U], dv[U];
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (ok[j]) {
                xv[j] = load_vec<T, V>(p.x.data, r * p.x.s0 + c[j]);
                dv[j] = load_vec<T, V>(p.dy.data, r * p.dy.s0 + c[j]);
            }
        float m1 = 0.0f, m2 = 0.0f;
        float xh[U][V], g[U][V];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (!ok[j]) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                xh[j][i] = (at<T, V>(xv[j], i) - mean) * rstd;
                const float du = at<T, V>(dv[j], i) * act_slope(fmaf(xh[j][i], w[j][i], b[j][i]), p.act);
                s1[j][i] += du;
                s2[j][i] = fmaf(du, xh[j][i], s2[j][i]);
                g[j][i] = du * w[j][i];
                m1 += g[j][i];
                m2 = fmaf(g[j][i], xh[j][i], m2);
            }
        }
        m1 = sum_lanes(m1, lg);
        m2 = sum_lanes(m2, lg);
        if (wpg != 1) {
            float(*slot)[4] = slots[((r - q.row0) / q.rstep) & 1];      // (the sums before these may still be read)
            if ((threadIdx.x & 63) == 0) slot[0][threadIdx.x >> 6] = m1, slot[1][threadIdx.x >> 6] = m2;
            __syncthreads();
            m1 = (slot[0][0] + slot[0][1]) + (slot[0][2] + slot[0][3]);
            m2 = (slot[1][0] + slot[1][1]) + (slot[1][2] + slot[1][3]);
        }
        m1 *= inv;
        m2 *= inv;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (!ok[j]) continue;
            vec_t<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) put<T, V>(o, i, rstd * (g[j][i] - m1 - xh[j][i] * m2));
            store_vec<T, V>(p.dx.data, r * p.dx.s0 + c[j], o);
        }
    }
    if (!p.dw && !p.db) return;
    float *out = p.part + (int64_t)blockIdx.y * 2 * p.C;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (wpg == 1) {         // the four wavefronts have the same columns
                __syncthreads();
#pragma unroll
                for (int i = 0; i < V; ++i) red[wave][lane][i] = k ? s2[j][i] : s1[j][i];
                __syncthreads();
                if (wave == 0 && ok[j])
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        out[k * p.C + c[j] + i] = (red[0][lane][i] + red[1][lane][i]) + (red[2][lane][i] + red[3][lane][i]);
            } else if (ok[j]) {
#pragma unroll
                for (int i = 0; i < V; ++i) out[k * p.C + c[j] + i] = k ? s2[j][i] : s1[j][i];
            }
        }
}

// ---------------------------------------------------------------------------
// chunks
// ---------------------------------------------------------------------------
// A workgroup has a row chunk of the columns of a tile: `groups` whole groups, or a piece of one that is wider than the
// workgroup.  Thread (row ty of rw, column tx of cols) keeps its column.
struct Tile {
    int g0, groups;        // first group, groups
    int piece, pieces;
    int cw, cols;          // columns of a group (of its piece), of the tile
    int rw, tx, ty;
    bool in;               // the thread has a column
    int c;                 // its first channel
    int64_t n, chunk, r0, r1;
};
template <int V> __device__ __forceinline__ Tile tile_of(const NormParams &p)
{
    const int cu = p.Cg / V;
    Tile t;
    // workgroups: column tiles of a chunk, chunks of an image, images (one number: an extent of the launch holds 65535 only)
    const uint32_t row = blockIdx.x / (uint32_t)p.ctiles;
    const int ct = (int)(blockIdx.x - row * (uint32_t)p.ctiles);
    const uint32_t n = row / (uint32_t)p.chunks;
    t.n = n;
    t.chunk = row - n * (uint32_t)p.chunks;
    t.pieces = (cu + NT - 1) / NT;
    if (t.pieces > 1) {
        t.g0 = ct / t.pieces;
        t.groups = 1;
        t.piece = ct - t.g0 * t.pieces;
        t.cw = min(NT, cu - t.piece * NT);
    } else {
        const int gt = p.group_tile;
        t.g0 = ct * gt;
        t.groups = min(gt, p.G - t.g0);
        t.piece = 0;
        t.cw = cu;
    }
    t.cols = t.groups * t.cw;
    t.rw = NT / t.cols;
    t.ty = (int)threadIdx.x / t.cols;
    t.tx = (int)threadIdx.x - t.ty * t.cols;
    t.in = t.ty < t.rw;
    t.c = t.g0 * p.Cg + (t.piece * NT + t.tx) * V;
    t.r0 = t.chunk * p.chunk_rows;
    t.r1 = min(t.r0 + p.chunk_rows, p.S);
    return t;
}

// (n, mean, m2) of two sets of values -> of both
__device__ __forceinline__ void join(float &n, float &mean, float &m2, float nb, float mb, float m2b)
{
    const float sum = n + nb, part = sum > 0.0f ? nb * __builtin_amdgcn_rcpf(sum) : 0.0f, d = mb - mean;
    mean = fmaf(d, part, mean);
    m2 += m2b + d * d * n * part;
    n = sum;
}

// over aligned runs of `lanes` (a power of two) lanes, in every one of them
__device__ __forceinline__ void join_lanes(float &n, float &mean, float &m2, int lanes)
{
#define MERIT_JOIN(BIT) if (lanes > 1 << BIT) join(n, mean, m2, lane_xor<BIT>(n), lane_xor<BIT>(mean), lane_xor<BIT>(m2));
    MERIT_JOIN(0) MERIT_JOIN(1) MERIT_JOIN(2) MERIT_JOIN(3) MERIT_JOIN(4) MERIT_JOIN(5)
#undef MERIT_JOIN
}
// threads (a power of two, at most a wavefront) that a workgroup has for each of its groups
__device__ __forceinline__ int group_lanes(int groups)
{
    int lanes = 64;
    while (lanes * groups > NT) lanes /= 2;
    return lanes;
}

// A value of the group, which the chunks' means are taken from: next to a mean that is far from zero their distances keep
// all digits
template <typename T> __device__ __forceinline__ float shift_of(const NormParams &p, int64_t n, int g)
{
    return (float)static_cast<const T *>(p.x.data)[n * p.x.s0 + (int64_t)g * p.Cg];
}

template <typename T, int V> __global__ __launch_bounds__(NT) void merit_norm_stats(NormParams p)
{
    __shared__ float sn[NT], sm[NT], sq[NT];
    const Tile t = tile_of<V>(p);
    const int64_t n = t.n, base = n * p.x.s0 + t.c;
    constexpr int RB = 4;                   // rows in flight
    float cnt = 0.0f, mean = 0.0f, m2 = 0.0f;
    if (t.in && t.r0 < t.r1) {
        const float k0 = shift_of<T>(p, n, t.g0 + t.tx / t.cw);
        int64_t r = t.r0 + t.ty, at0 = base + r * p.x.s1;
        const int64_t xs = t.rw * p.x.s1;
        for (; r + (RB - 1) * t.rw < t.r1; r += RB * t.rw) {
            vec_t<T, V> v[RB];
#pragma unroll
            for (int k = 0; k < RB; ++k, at0 += xs) v[k] = load_vec<T, V>(p.x.data, at0);
            float s = 0.0f, q = 0.0f;
#pragma unroll
            for (int k = 0; k < RB; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) s += at<T, V>(v[k], i) - k0;
            s *= 1.0f / (RB * V);
#pragma unroll
            for (int k = 0; k < RB; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = (at<T, V>(v[k], i) - k0) - s;
                    q = fmaf(d, d, q);
                }
            join(cnt, mean, m2, (float)(RB * V), s, q);
        }
        for (; r < t.r1; r += t.rw, at0 += xs) {
            const vec_t<T, V> v = load_vec<T, V>(p.x.data, at0);
            float s = 0.0f, q = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) s += at<T, V>(v, i) - k0;
            s *= 1.0f / V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = (at<T, V>(v, i) - k0) - s;
                q = fmaf(d, d, q);
            }
            join(cnt, mean, m2, (float)V, s, q);
        }
    }
    sn[threadIdx.x] = cnt;
    sm[threadIdx.x] = mean;
    sq[threadIdx.x] = m2;
    __syncthreads();
    const int lanes = group_lanes(t.groups), g = (int)threadIdx.x / lanes, lane = (int)threadIdx.x & (lanes - 1);
    cnt = mean = m2 = 0.0f;
    if (g < t.groups)
        for (int e = lane; e < t.rw * t.cw; e += lanes) {
            const int row = e / t.cw, k = row * t.cols + g * t.cw + (e - row * t.cw);
            join(cnt, mean, m2, sn[k], sm[k], sq[k]);
        }
    join_lanes(cnt, mean, m2, lanes);
    if (g < t.groups && lane == 0) {
        const int64_t parts = p.chunks * t.pieces;
        float *o = p.part + 2 * ((n * p.G + t.g0 + g) * parts + t.chunk * t.pieces + t.piece);
        o[0] = mean;
        o[1] = m2;
        // (kept for the second launch: its first workgroups may write over x)
        if (p.S > 0 && t.chunk == 0 && t.piece == 0) p.part[2 * p.N * p.G * parts + n * p.G + t.g0 + g] = shift_of<T>(p, n, t.g0 + g);
    }
}

// values of partial k of a group
template <int V> __device__ __forceinline__ float part_count(const NormParams &p, const Tile &t, int k)
{
    const int chunk = t.pieces == 1 ? k : k / t.pieces, cu = p.Cg / V;
    const int cw = t.pieces == 1 ? cu : min(NT, cu - (k - chunk * t.pieces) * NT);
    return (float)min((int)p.chunk_rows, (int)p.S - chunk * (int)p.chunk_rows) * (float)(cw * V);
}

template <typename T, int V> __global__ __launch_bounds__(NT) void merit_norm_apply(NormParams p)
{
    __shared__ float stat[NT][2];
    const Tile t = tile_of<V>(p);
    const int64_t n = t.n, parts = p.chunks * t.pieces;
    {
        const int lanes = group_lanes(t.groups), g = (int)threadIdx.x / lanes, lane = (int)threadIdx.x & (lanes - 1);
        float cnt = 0.0f, off = 0.0f, m2 = 0.0f;
        if (g < t.groups) {
            const float2 *in = reinterpret_cast<const float2 *>(p.part) + (n * p.G + t.g0 + g) * parts;
#pragma unroll 4
            for (int k = lane; k < (int)parts; k += lanes) {
                const float2 v = in[k];
                join(cnt, off, m2, part_count<V>(p, t, k), v.x, v.y);
            }
        }
        join_lanes(cnt, off, m2, lanes);
        if (g < t.groups && lane == 0) {
            const float mean = cnt > 0.0f ? p.part[2 * p.N * p.G * parts + n * p.G + t.g0 + g] + off : 0.0f;
            const float rstd = __builtin_amdgcn_rsqf((cnt > 0.0f ? m2 / cnt : 0.0f) + p.eps);
            stat[g][0] = mean;
            stat[g][1] = rstd;
            if (t.chunk == 0 && t.piece == 0) {
                if (p.mean) p.mean[n * p.G + t.g0 + g] = mean;
                if (p.rstd) p.rstd[n * p.G + t.g0 + g] = rstd;
            }
        }
    }
    __syncthreads();
    if (!t.in) return;
    const float mean = stat[t.tx / t.cw][0], rstd = stat[t.tx / t.cw][1];
    float w[V], b[V];
    load_params<T>(p.w, t.c, 1.0f, w);
    load_params<T>(p.b, t.c, 0.0f, b);
    const int64_t first = t.r0 + t.ty, xs = t.rw * p.x.s1, ys = t.rw * p.y.s1;
    int64_t xa = n * p.x.s0 + first * p.x.s1 + t.c, ya = n * p.y.s0 + first * p.y.s1 + t.c;
    constexpr int RB = 4;                   // rows in flight (y may be x: no load moves over a store by itself)
    for (int r = (int)first; r < (int)t.r1; r += RB * t.rw) {
        vec_t<T, V> v[RB];
        // (behind the last row: that one again; a load under a condition would be waited for before the next)
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            v[k] = load_vec<T, V>(p.x.data, xa);
            if (r + (k + 1) * t.rw < (int)t.r1) xa += xs;
        }
#pragma unroll
        for (int k = 0; k < RB; ++k, ya += ys) {
            if (k && r + k * t.rw >= (int)t.r1) break;
            vec_t<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) put<T, V>(o, i, apply_act(fmaf((at<T, V>(v[k], i) - mean) * rstd, w[i], b[i]), p.act));
            store_vec<T, V>(p.y.data, ya, o);
        }
    }
}

// per channel sum du, sum du xh; per group their sums with the weights
template <typename T, int V> __global__ __launch_bounds__(NT) void merit_norm_sums(NormParams p)
{
    __shared__ float red[2][NT][V];
    const Tile t = tile_of<V>(p);
    const int64_t n = t.n;
    float w[V], b[V], s1[V], s2[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s1[i] = s2[i] = 0.0f;
    if (t.in) {
        const int g = t.g0 + t.tx / t.cw;
        const float mean = p.mean[n * p.G + g], rstd = p.rstd[n * p.G + g];
        load_params<T>(p.w, t.c, 1.0f, w);
        load_params<T>(p.b, t.c, 0.0f, b);
        const int64_t first = t.r0 + t.ty, xs = t.rw * p.x.s1, ds = t.rw * p.dy.s1;
        int64_t xa = n * p.x.s0 + first * p.x.s1 + t.c, da = n * p.dy.s0 + first * p.dy.s1 + t.c;
#pragma unroll 4
        for (int r = (int)first; r < (int)t.r1; r += t.rw, xa += xs, da += ds) {
            const vec_t<T, V> xv = load_vec<T, V>(p.x.data, xa), dv = load_vec<T, V>(p.dy.data, da);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (at<T, V>(xv, i) - mean) * rstd;
                const float du = at<T, V>(dv, i) * act_slope(fmaf(xh, w[i], b[i]), p.act);
                s1[i] += du;
                s2[i] = fmaf(du, xh, s2[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        red[0][threadIdx.x][i] = s1[i];
        red[1][threadIdx.x][i] = s2[i];
    }
    __syncthreads();
    // the rows' sums, a thread for each channel and kind; they replace the first row's
    const int per = t.cols * V;
    float *out = p.part + (n * p.chunks + t.chunk) * 2 * p.C + t.g0 * p.Cg + t.piece * NT * V;
    for (int m = threadIdx.x; m < 2 * per; m += NT) {
        const int kind = m >= per, c = kind ? m - per : m;
        float *col = &red[kind][0][0] + c, s = col[0];
        for (int k = 1; k < t.rw; ++k) s += col[k * per];
        col[0] = s;
        out[kind * p.C + c] = s;
    }
    __syncthreads();
    const int lanes = group_lanes(t.groups), g = (int)threadIdx.x / lanes, lane = (int)threadIdx.x & (lanes - 1);
    float a = 0.0f, q = 0.0f;
    if (g < t.groups)
        for (int e = lane; e < t.cw * V; e += lanes) {
            const float wc = load_param<T>(p.w, (t.g0 + g) * p.Cg + t.piece * NT * V + e, 1.0f);
            a = fmaf(wc, (&red[0][0][0])[g * t.cw * V + e], a);
            q = fmaf(wc, (&red[1][0][0])[g * t.cw * V + e], q);
        }
    a = sum_lanes(a, lanes);
    q = sum_lanes(q, lanes);
    if (g < t.groups && lane == 0) {
        float *o = p.part + p.N * p.chunks * 2 * p.C + 2 * ((n * p.G + t.g0 + g) * p.chunks * t.pieces + t.chunk * t.pieces + t.piece);
        o[0] = a;
        o[1] = q;
    }
}

template <typename T, int V> __global__ __launch_bounds__(NT) void merit_norm_apply_backward(NormParams p)
{
    __shared__ float stat[NT][2];
    const Tile t = tile_of<V>(p);
    const int64_t n = t.n, parts = p.chunks * t.pieces;
    const float inv = 1.0f / ((float)p.S * (float)p.Cg);
    {
        const int lanes = group_lanes(t.groups), g = (int)threadIdx.x / lanes, lane = (int)threadIdx.x & (lanes - 1);
        float a = 0.0f, q = 0.0f;
        if (g < t.groups) {
            const float2 *in = reinterpret_cast<const float2 *>(p.part + p.N * p.chunks * 2 * p.C) + (n * p.G + t.g0 + g) * parts;
#pragma unroll 4
            for (int k = lane; k < (int)parts; k += lanes) {
                const float2 v = in[k];
                a += v.x;
                q += v.y;
            }
        }
        a = sum_lanes(a, lanes);
        q = sum_lanes(q, lanes);
        if (g < t.groups && lane == 0) {
            stat[g][0] = a * inv;
            stat[g][1] = q * inv;
        }
    }
    __syncthreads();
    if (!t.in) return;
    const int gl = t.tx / t.cw, g = t.g0 + gl;
    const float m1 = stat[gl][0], m2 = stat[gl][1], mean = p.mean[n * p.G + g], rstd = p.rstd[n * p.G + g];
    float w[V], b[V];
    load_params<T>(p.w, t.c, 1.0f, w);
    load_params<T>(p.b, t.c, 0.0f, b);
    const int64_t first = t.r0 + t.ty, xs = t.rw * p.x.s1, ds = t.rw * p.dy.s1, os = t.rw * p.dx.s1;
    int64_t xa = n * p.x.s0 + first * p.x.s1 + t.c, da = n * p.dy.s0 + first * p.dy.s1 + t.c,
            oa = n * p.dx.s0 + first * p.dx.s1 + t.c;
    constexpr int RB = 4;
    for (int r = (int)first; r < (int)t.r1; r += RB * t.rw) {
        vec_t<T, V> xv[RB], dv[RB];
#pragma unroll
        for (int k = 0; k < RB; ++k) {
            xv[k] = load_vec<T, V>(p.x.data, xa);
            dv[k] = load_vec<T, V>(p.dy.data, da);
            if (r + (k + 1) * t.rw < (int)t.r1) {
                xa += xs;
                da += ds;
            }
        }
#pragma unroll
        for (int k = 0; k < RB; ++k, oa += os) {
            if (k && r + k * t.rw >= (int)t.r1) break;
            vec_t<T, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float xh = (at<T, V>(xv[k], i) - mean) * rstd;
                const float g1 = at<T, V>(dv[k], i) * act_slope(fmaf(xh, w[i], b[i]), p.act) * w[i];
                put<T, V>(o, i, rstd * (g1 - m1 - xh * m2));
            }
            store_vec<T, V>(p.dx.data, oa, o);
        }
    }
}

// ---------------------------------------------------------------------------
// a group a workgroup
// ---------------------------------------------------------------------------
// All of a group's values of one image stay in the workgroup's registers, U units of V channels a thread: x (and dy) are
// read once and nothing waits for another workgroup.  (Eight units of eight channels in 1024 threads spill: 42 registers forward,
// 2 backward.)  Thread (row ty, unit tx) has rows ty, ty + rw, ...  A row of few
// channels fills less than a cache line; its neighbours in the line belong to workgroups that run on the same XCD.
struct Slab {
    int64_t n;
    int g, tx, ty, rw, c;
    bool in;
};
template <int V, int NTH> __device__ __forceinline__ Slab slab_of(const NormParams &p)
{
    const int cu = p.Cg / V;
    const uint32_t item = xcd_band_item(blockIdx.x, (int)(gridDim.x >> 3), (int)(gridDim.x & 7u)), n = item / (uint32_t)p.G;
    Slab s;
    s.n = n;
    s.g = (int)(item - n * (uint32_t)p.G);
    s.rw = NTH / cu;
    s.ty = (int)threadIdx.x / cu;
    s.tx = (int)threadIdx.x - s.ty * cu;
    s.c = s.g * p.Cg + s.tx * V;
    s.in = s.ty < s.rw;
    return s;
}
// the sum over a workgroup; `slot`: LDS of its own for every sum
template <int NTH> __device__ __forceinline__ float sum_block(float v, float *slot)
{
    v = sum_lanes(v, 64);
    if ((threadIdx.x & 63) == 0) slot[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < NTH / 64; ++i) s += slot[i];
    return s;
}

template <typename T, int V, int U, int NTH> __global__ __launch_bounds__(NTH) void merit_norm_slab(NormParams p)
{
    __shared__ float slots[2][NTH / 64];
    const Slab s = slab_of<V, NTH>(p);
    const int S = (int)p.S;
    vec_t<T, V> v[U];
    int64_t at0 = s.n * p.x.s0 + s.ty * p.x.s1 + s.c;
#pragma unroll
    for (int k = 0; k < U; ++k, at0 += s.rw * p.x.s1) {
        v[k] = vec_t<T, V>{};
        if (s.in && s.ty + k * s.rw < S) v[k] = load_vec<T, V>(p.x.data, at0);
    }
    float w[V], b[V];
    load_params<T>(p.w, s.in ? s.c : 0, 1.0f, w);
    load_params<T>(p.b, s.in ? s.c : 0, 0.0f, b);
    // distances from a value of the group: next to a mean that is far from zero they keep all digits
    const float k0 = shift_of<T>(p, s.n, s.g);
    float a = 0.0f, q = 0.0f;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const bool in = s.in && s.ty + k * s.rw < S;
#pragma unroll
        for (int i = 0; i < V; ++i) a += in ? at<T, V>(v[k], i) - k0 : 0.0f;
    }
    const float inv = 1.0f / ((float)S * (float)p.Cg), off = sum_block<NTH>(a, slots[0]) * inv, mean = k0 + off;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const bool in = s.in && s.ty + k * s.rw < S;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = in ? (at<T, V>(v[k], i) - k0) - off : 0.0f;
            q = fmaf(d, d, q);
        }
    }
    const float rstd = __builtin_amdgcn_rsqf(sum_block<NTH>(q, slots[1]) * inv + p.eps);
    if (threadIdx.x == 0) {
        if (p.mean) p.mean[s.n * p.G + s.g] = mean;
        if (p.rstd) p.rstd[s.n * p.G + s.g] = rstd;
    }
    int64_t yt = s.n * p.y.s0 + s.ty * p.y.s1 + s.c;
#pragma unroll
    for (int k = 0; k < U; ++k, yt += s.rw * p.y.s1) {
        if (!s.in || s.ty + k * s.rw >= S) continue;
        vec_t<T, V> o;
#pragma unroll
        for (int i = 0; i < V; ++i) put<T, V>(o, i, apply_act(fmaf((at<T, V>(v[k], i) - mean) * rstd, w[i], b[i]), p.act));
        store_vec<T, V>(p.y.data, yt, o);
    }
}

template <typename T, int V, int U, int NTH> __global__ __launch_bounds__(NTH) void merit_norm_slab_backward(NormParams p)
{
    __shared__ float slots[2][NTH / 64], red[NTH][V];
    const Slab s = slab_of<V, NTH>(p);
    const int S = (int)p.S;
    vec_t<T, V> xv[U], dv[U];
    int64_t xa = s.n * p.x.s0 + s.ty * p.x.s1 + s.c, da = s.n * p.dy.s0 + s.ty * p.dy.s1 + s.c;
#pragma unroll
    for (int k = 0; k < U; ++k, xa += s.rw * p.x.s1, da += s.rw * p.dy.s1) {
        xv[k] = dv[k] = vec_t<T, V>{};
        if (s.in && s.ty + k * s.rw < S) {
            xv[k] = load_vec<T, V>(p.x.data, xa);
            dv[k] = load_vec<T, V>(p.dy.data, da);
        }
    }
    const float mean = p.mean[s.n * p.G + s.g], rstd = p.rstd[s.n * p.G + s.g];
    float w[V], b[V], s1[V], s2[V];
    load_params<T>(p.w, s.in ? s.c : 0, 1.0f, w);
    load_params<T>(p.b, s.in ? s.c : 0, 0.0f, b);
#pragma unroll
    for (int i = 0; i < V; ++i) s1[i] = s2[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        if (!s.in || s.ty + k * s.rw >= S) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float xh = (at<T, V>(xv[k], i) - mean) * rstd;
            const float du = at<T, V>(dv[k], i) * act_slope(fmaf(xh, w[i], b[i]), p.act);
            s1[i] += du;
            s2[i] = fmaf(du, xh, s2[i]);
        }
    }
    float m1 = 0.0f, m2 = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        m1 = fmaf(w[i], s1[i], m1);
        m2 = fmaf(w[i], s2[i], m2);
    }
    const float inv = 1.0f / ((float)S * (float)p.Cg);
    m1 = sum_block<NTH>(s.in ? m1 : 0.0f, slots[0]) * inv;
    m2 = sum_block<NTH>(s.in ? m2 : 0.0f, slots[1]) * inv;
    int64_t ot = s.n * p.dx.s0 + s.ty * p.dx.s1 + s.c;
#pragma unroll
    for (int k = 0; k < U; ++k, ot += s.rw * p.dx.s1) {
        if (!s.in || s.ty + k * s.rw >= S) continue;
        vec_t<T, V> o;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float xh = (at<T, V>(xv[k], i) - mean) * rstd;
            const float g1 = at<T, V>(dv[k], i) * act_slope(fmaf(xh, w[i], b[i]), p.act) * w[i];
            put<T, V>(o, i, rstd * (g1 - m1 - xh * m2));
        }
        store_vec<T, V>(p.dx.data, ot, o);
    }
    if (!p.dw && !p.db) return;
    // the rows' sums of a channel
    float *out = p.part + s.n * 2 * p.C + s.g * p.Cg;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        if (kind) __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) red[threadIdx.x][i] = kind ? s2[i] : s1[i];
        __syncthreads();
        // a wavefront for each channel in turn
        for (int c = threadIdx.x >> 6; c < p.Cg; c += NTH / 64) {
            const int u = c / V, i = c - u * V, cu = p.Cg / V;
            float v = 0.0f;
            for (int r = threadIdx.x & 63; r < s.rw; r += 64) v += red[r * cu + u][i];
            v = sum_lanes(v, 64);
            if ((threadIdx.x & 63) == 0) out[kind * p.C + c] = v;
        }
    }
}

// ---------------------------------------------------------------------------
// sums over workgroups' partial results
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(1024) void merit_reduce_rows(ReduceParams p)
{
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t j = (int64_t)blockIdx.x * 64 + lane;
    int k = 0;
    while (k < p.nseg - 1 && j >= p.seg[k].len) j -= p.seg[k].len, ++k;
    const bool in = j < p.seg[k].len && p.seg[k].out;
    float s = 0.0f;
    if (in) {
        const float *col = p.in + p.seg[k].at + j;
#pragma unroll 8
        for (int64_t r = wave; r < p.rows; r += 16) s += col[r * p.pitch];
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && in) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += red[i][lane];
        p.seg[k].out[j] = s;
    }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------
struct RowsForm {
    int cu, lg, wpg, U;
};
RowsForm norm_rows_form(const NormParams &p)
{
    RowsForm f;
    f.cu = p.Cg / p.vec;
    f.wpg = f.cu > 256 ? 4 : 1;
    f.lg = 1;
    while (f.lg < 64 && f.lg < f.cu) f.lg *= 2;
    const int per = (f.cu + f.lg * f.wpg - 1) / (f.lg * f.wpg);
    f.U = per <= 1 ? 1 : per <= 2 ? 2 : 4;
        return f;
}

template <typename T, int V> hipError_t norm_forward(const NormParams &p, hipStream_t s)
{
    if (p.rows_form) {
        const RowsForm f = norm_rows_form(p);
        const dim3 grid(p.ctiles, (unsigned)p.chunks);
        if (f.U == 1) merit_norm_rows<T, V, 1><<<grid, NT, 0, s>>>(p, f.cu, f.lg, f.wpg);
        else if (f.U == 2) merit_norm_rows<T, V, 2><<<grid, NT, 0, s>>>(p, f.cu, f.lg, f.wpg);
        else merit_norm_rows<T, V, 4><<<grid, NT, 0, s>>>(p, f.cu, f.lg, f.wpg);
        return hipGetLastError();
    }
    if constexpr (V > 1)
        if (p.slab) {
            const unsigned grid = (unsigned)(p.N * p.G);
            switch (p.slab) {
            case 0x104: merit_norm_slab<T, V, 4, 256><<<grid, 256, 0, s>>>(p); break;
            case 0x108: merit_norm_slab<T, V, 8, 256><<<grid, 256, 0, s>>>(p); break;
            case 0x404: merit_norm_slab<T, V, 4, 1024><<<grid, 1024, 0, s>>>(p); break;
            default: merit_norm_slab<T, V, 8, 1024><<<grid, 1024, 0, s>>>(p); break;
            }
            return hipGetLastError();
        }
    const unsigned grid = (unsigned)(p.N * p.chunks * p.ctiles);
    merit_norm_stats<T, V><<<grid, NT, 0, s>>>(p);
    merit_norm_apply<T, V><<<grid, NT, 0, s>>>(p);
    return hipGetLastError();
}

template <typename T, int V> hipError_t norm_backward(const NormParams &p, hipStream_t s)
{
    int64_t rows;
    if (p.rows_form) {
        const RowsForm f = norm_rows_form(p);
        const dim3 grid(p.ctiles, (unsigned)p.chunks);
        if (f.U == 1) merit_norm_rows_backward<T, V, 1><<<grid, NT, 0, s>>>(p, f.cu, f.lg, f.wpg);
        else if (f.U == 2) merit_norm_rows_backward<T, V, 2><<<grid, NT, 0, s>>>(p, f.cu, f.lg, f.wpg);
        else merit_norm_rows_backward<T, V, 4><<<grid, NT, 0, s>>>(p, f.cu, f.lg, f.wpg);
        rows = p.chunks;
    } else if (V > 1 && p.slab) {
        const unsigned grid = (unsigned)(p.N * p.G);
        if constexpr (V > 1) switch (p.slab) {
            case 0x104: merit_norm_slab_backward<T, V, 4, 256><<<grid, 256, 0, s>>>(p); break;
            case 0x108: merit_norm_slab_backward<T, V, 8, 256><<<grid, 256, 0, s>>>(p); break;
            case 0x404: merit_norm_slab_backward<T, V, 4, 1024><<<grid, 1024, 0, s>>>(p); break;
            default: merit_norm_slab_backward<T, V, 8, 1024><<<grid, 1024, 0, s>>>(p); break;
            }
        rows = p.N;
    } else {
        const unsigned grid = (unsigned)(p.N * p.chunks * p.ctiles);
        merit_norm_sums<T, V><<<grid, NT, 0, s>>>(p);
        merit_norm_apply_backward<T, V><<<grid, NT, 0, s>>>(p);
        rows = p.N * p.chunks;
    }
    if (p.dw || p.db) {
        ReduceParams r = {};
        r.in = p.part;
        r.rows = rows;
        r.pitch = 2ll * p.C;
        r.nseg = 2;
        r.seg[0] = {p.db, 0, p.C};
        r.seg[1] = {p.dw, p.C, p.C};
        return launch_reduce_rows(r, s);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_reduce_rows(const ReduceParams &p, hipStream_t s)
{
    int64_t cols = 0;
    for (int k = 0; k < p.nseg; ++k) cols += p.seg[k].len;
    merit_reduce_rows<<<(unsigned)((cols + 63) / 64), 1024, 0, s>>>(p);
    return hipGetLastError();
}

namespace {

template <bool BACKWARD, typename T, int V> hipError_t norm_pass(const NormParams &p, hipStream_t s)
{
    if constexpr (BACKWARD) return norm_backward<T, V>(p, s);
    else return norm_forward<T, V>(p, s);
}
template <bool BACKWARD, typename T> hipError_t norm_typed(const NormParams &p, hipStream_t s)
{
    if constexpr (sizeof(T) == 2)
        if (p.vec == 8) return norm_pass<BACKWARD, T, 8>(p, s);
    if (p.vec == 4) return norm_pass<BACKWARD, T, 4>(p, s);
    return p.vec == 2 ? norm_pass<BACKWARD, T, 2>(p, s) : norm_pass<BACKWARD, T, 1>(p, s);
}
template <bool BACKWARD> hipError_t norm_any(const NormParams &p, int type, hipStream_t s)
{
    if (type == MERIT_F32) return norm_typed<BACKWARD, float>(p, s);
    return type == MERIT_F16 ? norm_typed<BACKWARD, f16_t>(p, s) : norm_typed<BACKWARD, bf16_t>(p, s);
}

}  // namespace

hipError_t launch_norm(const NormParams &p, int type, hipStream_t s) { return norm_any<false>(p, type, s); }
hipError_t launch_norm_backward(const NormParams &p, int type, hipStream_t s) { return norm_any<true>(p, type, s); }

}  // namespace merit
