// Device helpers of the gated delta rule's kernels (delta.hip, delta_backward.hip).
//
//     S_t = a_t S_{t-1} + k_t u_t^T,   u_t = b_t d_t,   d_t = v_t - a_t S_{t-1}^T k_t,   y_t = scale S_t^T q_t,   a_t = exp(g_t)
//
// A chunk of C = 64 tokens at once, G_t = g_1 + .. + g_t inside it, f_tj = exp(G_t - G_j), N_tj = f_tj k_t.k_j below the diagonal:
//     (1 + N diag(b)) d = r = v - exp(G) K S_0,    y = scale (exp(G) Q S_0 + (f o Q K^T) u),    S_C = exp(G_C) S_0 + K^T (exp(G_C - G) u)
// so that a token's dependence on those before it is a triangular matrix, and the rest are matrix products.  With
//     W = (1 + N diag(b))^-1 N,   (1 + N diag(b))^-1 = 1 - W diag(b),   (1 + diag(b) N)^-1 = 1 - diag(b) W
// one matrix serves the forward pass, d = r - W (b r), and the backward pass, x = y - W^T (b y), whatever b is (0 too).
// merit_delta_prepare finds it and P = scale f o Q K^T for all chunks side by side.
//
// Products run on v_mfma_f32_16x16x32_bf16.  An fp32 operand goes in as three bfloat16 terms of 8 bits each (x = x0 + x1 + x2 with
// the rounding error of the one before in each), a binary16 one as two, a bfloat16 one as it is, and terms whose product is below
// 2^-24 of the leading one are left out: 3 products for an exact operand with an fp32 one, 6 for two fp32 ones, at a sixteenth of
// the time each that v_mfma_f32_16x16x4_f32 takes.  States, sums and what is kept of them are fp32.
#pragma once

#include <type_traits>

#include "merit_internal.h"
#include "tokens.h"

namespace merit {
namespace delta {

constexpr int C = MERIT_DELTA_CHUNK;
constexpr int NT = 256;
static_assert(C == 64, "a wavefront has 16 of a chunk's tokens, a lane one of its decays");

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// bfloat16 terms that hold a value of type T
template <typename T> struct Terms { static constexpr int n = 3; };
template <> struct Terms<f16_t> { static constexpr int n = 2; };
template <> struct Terms<bf16_t> { static constexpr int n = 1; };

// Terms of P and u where they give y, which is rounded to T: two leave 2^-17, next to the 2^-12 of a rounding to binary16 (the
// gradients that P gives go on into sums in fp32: three)
template <typename T> constexpr int mix_terms() { return Terms<T>::n == 3 ? 3 : 2; }

template <int N> __device__ __forceinline__ void split(float x, __bf16 (&o)[N])
{
    o[0] = (__bf16)x;
#pragma unroll
    for (int i = 1; i < N; ++i) {
        x -= (float)o[i - 1];
        o[i] = (__bf16)x;
    }
}
template <int N> __device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&o)[N])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        __bf16 t[N];
        split<N>(x[e], t);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i][e] = t[i];
    }
}

// acc += a b over the pairs of terms (i, j) with i + j < ORDER, the small ones first
template <int ORDER, int NA, int NB>
__device__ __forceinline__ void multiply(f32x4 &acc, const bf16x8 (&a)[NA], const bf16x8 (&b)[NB])
{
#pragma unroll
    for (int s = ORDER - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = s - i;
            if (j >= 0 && j < NB) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[j], acc, 0, 0, 0);
        }
}

// The same for columns side by side, one after the other in turn: a product into an accumulator waits for the one before it
template <int ORDER, int NA, int NB, int NC>
__device__ __forceinline__ void multiply(f32x4 (&acc)[NC], const bf16x8 (&a)[NA], const bf16x8 (&b)[NC][NB])
{
#pragma unroll
    for (int s = ORDER - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = s - i;
            if (j >= 0 && j < NB)
#pragma unroll
                for (int c = 0; c < NC; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[c][j], acc[c], 0, 0, 0);
        }
}

// And for rows
template <int ORDER, int NA, int NB, int NR>
__device__ __forceinline__ void multiply_rows(f32x4 (&acc)[NR], const bf16x8 (&a)[NR][NA], const bf16x8 (&b)[NB])
{
#pragma unroll
    for (int s = ORDER - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = s - i;
            if (j >= 0 && j < NB)
#pragma unroll
                for (int r = 0; r < NR; ++r) acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[r][i], b[j], acc[r], 0, 0, 0);
        }
}

// ---- operands -----------------------------------------------------------------------------------------------
// Eight values of a row from column c on, zeros from column n on.  wide: rows start on 16 bytes and n is a multiple of 8.
template <typename T> struct Eight {
    typedef T vec __attribute__((ext_vector_type(8)));      // (16-bit values stay two in a register)
    vec v;
};
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x8 __attribute__((ext_vector_type(8)));
template <typename T> __device__ __forceinline__ Eight<T> zero8()
{
    Eight<T> r;
    if constexpr (sizeof(T) == 2) r.v = __builtin_bit_cast(typename Eight<T>::vec, u32x4{0, 0, 0, 0});
    else r.v = __builtin_bit_cast(typename Eight<T>::vec, u32x8{0, 0, 0, 0, 0, 0, 0, 0});
    return r;
}
template <typename T> __device__ __forceinline__ Eight<T> load8(const T *row, int c, int n, bool wide)
{
    Eight<T> r = zero8<T>();
    if (wide) {
        if (c < n) {
            const u32x4 *from = reinterpret_cast<const u32x4 *>(row + c);
            if constexpr (sizeof(T) == 2) {
                r.v = __builtin_bit_cast(typename Eight<T>::vec, from[0]);
            } else {
                const u32x4 a = from[0], b = from[1];
                r.v = __builtin_bit_cast(typename Eight<T>::vec, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < n) r.v[e] = row[c + e];
    }
    return r;
}
template <typename T> __device__ __forceinline__ void terms8(const Eight<T> &x, bf16x8 (&o)[Terms<T>::n])
{
    if constexpr (Terms<T>::n == 1) {
        o[0] = x.v;
    } else {
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)x.v[e];
        split8<Terms<T>::n>(f, o);
    }
}

// A matrix in LDS: planes of bfloat16 terms, rows of COLS values and 16 bytes more (16 rows of 16 bytes then lie in all banks)
template <int PLANES, int ROWS, int COLS> struct Tile {
    static constexpr int pitch = COLS + 8;
    static constexpr int plane = ROWS * pitch;
    __bf16 *at;
    static constexpr int bytes = PLANES * plane * 2;

    // Operand of a product whose sum runs along the rows of this matrix: lane l has row r0 + l % 16, columns c0 + 8 (l / 16) ..
    template <int N = PLANES> __device__ __forceinline__ void rows(int r0, int c0, bf16x8 (&o)[N]) const
    {
        const int lane = threadIdx.x & 63;
        const __bf16 *p = at + (r0 + (lane & 15)) * pitch + c0 + 8 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = *reinterpret_cast<const bf16x8 *>(p + i * plane);
    }
    // Operand of a product whose sum runs down the columns: lane l has column c0 + l % 16, rows r0 + 8 (l / 16) ..  A transposing
    // read takes four rows of 16 columns from 16 lanes, each of which names 8 bytes, and leaves lane i the i-th column.
    template <int N = PLANES> __device__ __forceinline__ void cols(int r0, int c0, bf16x8 (&o)[N]) const
    {
        typedef short short4v __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) short4v *lds4;
        const int lane = threadIdx.x & 63;
        const __bf16 *p = at + (r0 + 8 * (lane >> 4) + ((lane & 15) >> 2)) * pitch + c0 + 4 * (lane & 3);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + i * plane));
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + i * plane + 4 * pitch));
            o[i] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
    // Four values side by side in a row
    __device__ __forceinline__ void put4(int r, int c, const float (&x)[4]) const
    {
        bf16x4 o[PLANES];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            __bf16 t[PLANES];
            split<PLANES>(x[e], t);
#pragma unroll
            for (int i = 0; i < PLANES; ++i) o[i][e] = t[i];
        }
#pragma unroll
        for (int i = 0; i < PLANES; ++i) *reinterpret_cast<bf16x4 *>(at + i * plane + r * pitch + c) = o[i];
    }
    __device__ __forceinline__ void put1(int r, int c, float x) const
    {
        __bf16 t[PLANES];
        split<PLANES>(x, t);
#pragma unroll
        for (int i = 0; i < PLANES; ++i) at[i * plane + r * pitch + c] = t[i];
    }
    __device__ __forceinline__ void put8(int r, int c, const bf16x8 (&o)[PLANES]) const
    {
#pragma unroll
        for (int i = 0; i < PLANES; ++i) *reinterpret_cast<bf16x8 *>(at + i * plane + r * pitch + c) = o[i];
    }
    __device__ __forceinline__ float value(int r, int c) const
    {
        float x = 0.0f;
#pragma unroll
        for (int i = PLANES - 1; i >= 0; --i) x += (float)at[i * plane + r * pitch + c];
        return x;
    }
};

// The same with every 32 columns in the order in which two results of 16 x 16, one under the other, lie in a lane: 8 values side by
// side are 4 q .. 4 q + 3 of the first 16 and of the second.  A product then takes results as they come out of other products
// (`operand`): what a wavefront computes for its columns never leaves its registers.
__device__ __forceinline__ int interleaved(int c) { return (c & ~31) + 8 * ((c & 15) >> 2) + 4 * ((c >> 4) & 1) + (c & 3); }
template <int PLANES, int COLS> struct Mixed {
    static constexpr int pitch = COLS + 8;
    static constexpr int plane = C * pitch;
    static constexpr int bytes = PLANES * plane * 2;
    __bf16 *at;

    // Sums along the rows: lane l has row 16 rt + l % 16 and the 32 columns of f
    __device__ __forceinline__ void rows(int rt, int f, bf16x8 (&o)[PLANES]) const
    {
        const int lane = threadIdx.x & 63;
        const __bf16 *p = at + (16 * rt + (lane & 15)) * pitch + 32 * f + 8 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < PLANES; ++i) o[i] = *reinterpret_cast<const bf16x8 *>(p + i * plane);
    }
    // Sums down the columns: lane l has column 16 ct + l % 16 and the 32 rows of f, in results' order.  A transposing read takes
    // four rows of 16 columns from 16 lanes, each of which names 8 bytes, and leaves lane i the i-th column.
    __device__ __forceinline__ void cols(int f, int ct, bf16x8 (&o)[PLANES]) const
    {
        typedef short short4v __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) short4v *lds4;
        const int lane = threadIdx.x & 63;
        const __bf16 *p = at + (32 * f + 4 * (lane >> 4) + ((lane & 15) >> 2)) * pitch + 32 * (ct >> 1) + 8 * (lane & 3) + 4 * (ct & 1);
#pragma unroll
        for (int i = 0; i < PLANES; ++i) {
            const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + i * plane));
            const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + i * plane + 16 * pitch));
            o[i] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
    // Columns c .. c + 7 of a row
    __device__ __forceinline__ void put8(int r, int c, const bf16x8 (&o)[PLANES]) const
    {
        __bf16 *p = at + r * pitch + interleaved(c);
#pragma unroll
        for (int i = 0; i < PLANES; ++i) {
            *reinterpret_cast<bf16x4 *>(p + i * plane) = __builtin_shufflevector(o[i], o[i], 0, 1, 2, 3);
            *reinterpret_cast<bf16x4 *>(p + i * plane + 8) = __builtin_shufflevector(o[i], o[i], 4, 5, 6, 7);
        }
    }
};
// Two results of 16 x 16, one under the other, as an operand whose sum runs down their rows
template <int N> __device__ __forceinline__ void operand(const f32x4 &top, const f32x4 &bottom, bf16x8 (&o)[N])
{
    const float x[8] = {top[0], top[1], top[2], top[3], bottom[0], bottom[1], bottom[2], bottom[3]};
    split8<N>(x, o);
}

// A triangular matrix of C x C in terms, as merit_delta_prepare leaves it: its columns interleaved, of the upper half of its rows the
// left half.
__device__ __forceinline__ int triangle_at(int t, int c) { return t < C / 2 ? t * (C / 2) + c : C * C / 4 + (t - C / 2) * C + c; }
constexpr int TRIANGLE = C * C * 3 / 4;
// The first PLANES of its terms on their way into LDS
template <int PLANES> struct Triangle {
    static constexpr int per = TRIANGLE / 8, all = PLANES * per, units = (all + NT - 1) / NT;
    bf16x8 e[units];
    __device__ __forceinline__ void load(const __bf16 *from)
    {
#pragma unroll
        for (int i = 0; i < units; ++i) {
            const int u = (int)threadIdx.x + i * NT;
            e[i] = reinterpret_cast<const bf16x8 *>(from)[u < all ? u : all - 1];
        }
    }
    __device__ __forceinline__ void store(const Mixed<PLANES, C> &t) const
    {
#pragma unroll
        for (int i = 0; i < units; ++i) {
            const int u = (int)threadIdx.x + i * NT, v = u % per, w = v - per / 3;
            const int at = v < per / 3 ? (v >> 2) * t.pitch + (v & 3) * 8 : (C / 2 + (w >> 3)) * t.pitch + (w & 7) * 8;
            if (u < all) *reinterpret_cast<bf16x8 *>(t.at + u / per * t.plane + at) = e[i];
        }
    }
};
// What merit_delta_prepare leaves of a chunk of a head
struct Prepared {
    __bf16 *w, *mix;        // -W and P, three terms each (of P two, where nothing but y of a 16-bit type is made of it)
    float *scal;
};
constexpr int PREPARED_FLOATS = DELTA_PREPARED_FLOATS;
static_assert(PREPARED_FLOATS == 3 * TRIANGLE + DELTA_SCALAR_FLOATS, "");
__device__ __forceinline__ Prepared prepared(const DeltaParams &p, int64_t chunk)
{
    float *at = p.prep + chunk * p.prep_stride;
    Prepared r;
    r.scal = at;
    r.w = reinterpret_cast<__bf16 *>(at + DELTA_SCALAR_FLOATS);
    r.mix = r.w + 3 * TRIANGLE;
    return r;
}

// Eight values of a row of n, from column c on, zeros from column n on; nothing stands in a branch, so that loads of many rows go out
// together.  WIDE: rows start on 16 bytes and n is a multiple of 8.
template <bool WIDE, typename T> __device__ __forceinline__ Eight<T> take8(const T *row, int c, int n)
{
    Eight<T> r;
    if constexpr (WIDE) {
        const u32x4 *from = reinterpret_cast<const u32x4 *>(row + (c < n ? c : 0));
        if constexpr (sizeof(T) == 2) {
            u32x4 a = from[0];
            if (c >= n) a = u32x4{0, 0, 0, 0};
            r.v = __builtin_bit_cast(typename Eight<T>::vec, a);
        } else {
            u32x4 a = from[0], b = from[1];
            if (c >= n) a = b = u32x4{0, 0, 0, 0};
            r.v = __builtin_bit_cast(typename Eight<T>::vec, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const T x = row[max(min(c + e, n - 1), 0)];        // (n may be 0: a row of zeros, of which the first value is there)
            r.v[e] = c + e < n ? x : (T)0.0f;
        }
    }
    return r;
}

// A chunk's rows of q or k: unit u of a thread is row u / (KF * 4) of the tile and eight columns.  FULL: all C rows are there, else m,
// at least one, the others zeros.
template <typename T, int KF> struct ChunkRows {
    static constexpr int units = C * KF * 4 / NT, step = NT / (KF * 4);
    Eight<T> e[units];

    template <bool FULL, bool WIDE>
    __device__ __forceinline__ void load(const Rows &x, int64_t b, int64_t t0, int m, int head, int D)
    {
        const int r0 = (int)threadIdx.x / (KF * 4), c = (int)threadIdx.x % (KF * 4) * 8;
        const T *from = static_cast<const T *>(x.data) + b * x.s0 + t0 * x.s1 + (int64_t)head * D;
        const T *row = from + r0 * x.s1;
#pragma unroll
        for (int i = 0; i < units; ++i) {
            if constexpr (FULL) {
                e[i] = take8<WIDE, T>(row + i * step * x.s1, c, D);
            } else {
                const int r = r0 + i * step;
                e[i] = take8<WIDE, T>(from + min(r, m - 1) * x.s1, c, r < m ? D : 0);
            }
        }
    }
    template <typename M> __device__ __forceinline__ void store(const M &t) const
    {
#pragma unroll
        for (int i = 0; i < units; ++i) {
            const int u = (int)threadIdx.x + i * NT;
            bf16x8 o[Terms<T>::n];
            terms8<T>(e[i], o);
            t.put8(u / (KF * 4), u % (KF * 4) * 8, o);
        }
    }
};

// A lane's sixteen values of a column of v or dy, in the order of four results one under the other
template <typename T> struct ChunkColumn {
    T v[C / 16][4];

    // `c`: a column that is there
    template <bool FULL> __device__ __forceinline__ void load(const Rows &x, int64_t b, int64_t t0, int m, int64_t c)
    {
        const int quad = (threadIdx.x & 63) >> 4;
        const T *from = static_cast<const T *>(x.data) + b * x.s0 + t0 * x.s1 + c, *row = from + 4 * quad * x.s1;
#pragma unroll
        for (int rt = 0; rt < C / 16; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (FULL) {
                    v[rt][r] = row[(16 * rt + r) * x.s1];
                } else {
                    const int t = 16 * rt + 4 * quad + r;
                    const T f = from[min(t, m - 1) * x.s1];
                    v[rt][r] = t < m ? f : (T)0.0f;
                }
            }
    }
};
// Sixteen results to a column of `x`: tokens from m on are zeros, those from `there` on are not
template <bool FULL, typename T>
__device__ __forceinline__ void put_column(const f32x4 (&v)[C / 16], const Rows &x, int64_t b, int64_t t0, int m, int there, int64_t c, bool in)
{
    const int quad = (threadIdx.x & 63) >> 4;
    T *row = static_cast<T *>(x.data) + b * x.s0 + (t0 + 4 * quad) * x.s1 + c;
    if (in)
#pragma unroll
        for (int rt = 0; rt < C / 16; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 16 * rt + 4 * quad + r;
                if (FULL || t < there) row[(16 * rt + r) * x.s1] = (T)(FULL || t < m ? v[rt][r] : 0.0f);
            }
}
// A wavefront's 16 columns of a state, rows of Dv
template <int DT> __device__ __forceinline__ void put_state(const f32x4 (&S)[DT], float *out, int Dk, int64_t Dv, bool in)
{
    const int quad = (threadIdx.x & 63) >> 4;
    float *row = out + 4 * quad * Dv;
    if (!in) return;
    if (Dk == 16 * DT) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) row[(16 * d + r) * Dv] = S[d][r];
    } else {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * d + 4 * quad + r < Dk) row[(16 * d + r) * Dv] = S[d][r];
    }
}

// What merit_delta_prepare leaves of a chunk of a head, 64 values each
enum { IN_K = 0,        // exp(G) / |k|
       BETA = 1,
       OUT_K = 2,       // exp(G_C - G) / |k|
       IN_Q = 3,        // scale exp(G) / |q|
       INV_K = 4, INV_Q = 5,                    // 1 / |k|, 1 / |q| (1 where they are taken as they are)
       SCALARS = 6 };
constexpr int SCALAR_FLOATS = DELTA_SCALAR_FLOATS;      // and G in 64 bits behind them
static_assert(SCALAR_FLOATS == SCALARS * C + 2 * C, "");

__device__ __forceinline__ int tokens_of(const DeltaParams &p, int64_t b)
{
    return p.lens ? min(max((int)p.lens[b], 0), (int)p.L) : (int)p.L;
}
// exp(x) of a difference of two 64-bit sums
__device__ __forceinline__ float exp_of(double x) { return __builtin_amdgcn_exp2f((float)(x * 1.44269504088896340736)); }

}  // namespace delta
}  // namespace merit
