// Device helpers of the gated delta rule's kernels (delta_forward.h, delta_backward.h).
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
// Products run on v_mfma_f32_16x16x32_bf16.  An fp32 operand goes in as three bfloat16 terms of 8 bits each (x = x0 + x1 + x2, each
// what the ones before it leave), a binary16 one as two, a bfloat16 one as it is: 3 products for a bfloat16 operand with an fp32
// one, 5 for a binary16 one, 6 for two fp32 ones, at a sixteenth of the time each that v_mfma_f32_16x16x4_f32 takes.  Of the others
// each is at most 2^-23 of the whole and of either sign (`split8`), so that sums are off by as much as those of fp32 products
// rounded one by one.  (Below 2^-110 a value's third term has fewer than 8 bits: bfloat16 ends at 2^-133.)  States, sums and what is
// kept of them are fp32.
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

template <int N> __device__ __forceinline__ void split(float x, __bf16 (&o)[N])
{
    o[0] = (__bf16)x;
#pragma unroll
    for (int i = 1; i < N; ++i) {
        x -= (float)o[i - 1];
        o[i] = (__bf16)x;
    }
}
// Eight values side by side.  Three terms of 8 bits each are the value itself (24 bits).  The first is cut off, so that it is never
// beyond the largest value, the second is rounded to the nearest: the third then has either sign, and so have the products that
// `multiply` leaves out, each at most 2^-23 of the whole (with the second cut off too, 2^-22, all of the product's own sign).
template <int N> __device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&o)[N])
{
    if constexpr (N == 3) {
        unsigned w[3][4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float a = x[e], b = x[e + 1];
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                unsigned ua = __builtin_bit_cast(unsigned, a), ub = __builtin_bit_cast(unsigned, b);
                if (i == 1) {
                    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                    w[1][e / 2] = __builtin_bit_cast(unsigned, (bf16x2){(__bf16)a, (__bf16)b});
                    ua = w[1][e / 2] << 16;
                    ub = w[1][e / 2];
                } else {
                    w[i][e / 2] = __builtin_amdgcn_perm(ub, ua, 0x07060302);       // the upper halves of both
                }
                if (i < 2) {
                    a -= __builtin_bit_cast(float, ua & 0xFFFF0000u);
                    b -= __builtin_bit_cast(float, ub & 0xFFFF0000u);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) __builtin_memcpy(&o[i], w[i], 16);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            __bf16 t[N];
            split<N>(x[e], t);
#pragma unroll
            for (int i = 0; i < N; ++i) o[i][e] = t[i];
        }
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

// The same for rows side by side, one after the other in turn: a product into an accumulator waits for the one before it
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
// Eight values of a row
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

// Products of chunks.  Row i of a result of 16 x 16 stands for token (or key value) 32 h + 8 (i / 4) + 4 s + i % 4: of two results, s = 0
// and 1, a lane then has eight that follow each other, which is how it has to have them for a sum along them (`operand`).  What a
// wavefront computes for its columns so goes from product to product in its registers; the other operands' rows are read in that
// order from LDS, where they lie as in memory.
__device__ __forceinline__ int row_of(int half, int sub) { const int i = threadIdx.x & 15; return 32 * half + 8 * (i >> 2) + 4 * sub + (i & 3); }

// Two results of 16 x 16 as an operand whose sum runs down their rows
template <int N> __device__ __forceinline__ void operand(const f32x4 &s0, const f32x4 &s1, bf16x8 (&o)[N])
{
    const float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
    split8<N>(x, o);
}
// A transposing read takes four rows of 16 columns from 16 lanes, each of which names 8 bytes (row i / 4, columns 4 (i % 4) ..), and leaves
// lane i the i-th column.
__device__ __forceinline__ bf16x8 transposed(const __bf16 *lo, const __bf16 *hi)
{
    typedef short short4v __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) short4v *lds4;
    const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)lo), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)hi);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A chunk's keys or queries in LDS
template <int PLANES, int COLS> struct Keys {
    static constexpr int pitch = COLS + 8, plane = C * pitch, bytes = PLANES * plane * 2;
    __bf16 *at;

    // tokens of (half, sub), the 32 columns of f
    __device__ __forceinline__ void rows(int half, int sub, int f, bf16x8 (&o)[PLANES]) const
    {
        const __bf16 *p = at + row_of(half, sub) * pitch + 32 * f + 8 * ((threadIdx.x & 63) >> 4);
#pragma unroll
        for (int i = 0; i < PLANES; ++i) o[i] = *reinterpret_cast<const bf16x8 *>(p + i * plane);
    }
    // columns of (f, sub), the 32 tokens of `half`
    __device__ __forceinline__ void cols(int f, int sub, int half, bf16x8 (&o)[PLANES]) const
    {
        const int lane = threadIdx.x & 63;
        const __bf16 *p = at + (32 * half + 8 * (lane >> 4) + ((lane & 15) >> 2)) * pitch + 32 * f + 8 * (lane & 3) + 4 * sub;
#pragma unroll
        for (int i = 0; i < PLANES; ++i) o[i] = transposed(p + i * plane, p + i * plane + 4 * pitch);
    }
    __device__ __forceinline__ void put8(int r, int c, const bf16x8 (&o)[PLANES]) const
    {
#pragma unroll
        for (int i = 0; i < PLANES; ++i) *reinterpret_cast<bf16x8 *>(at + i * plane + r * pitch + c) = o[i];
    }
};

// A triangular matrix of C x C: of the upper half of its rows the left half
__device__ __forceinline__ int triangle_at(int t, int c) { return t < C / 2 ? t * (C / 2) + c : C * C / 4 + (t - C / 2) * C + c; }
constexpr int TRIANGLE = C * C * 3 / 4;
// in LDS
template <int PLANES> struct Triangle {
    static constexpr int upper = C / 2 + 8, lower = C + 8, plane = C / 2 * (upper + lower), bytes = PLANES * plane * 2;
    __bf16 *at;

    static __device__ __forceinline__ int line(int half, int r) { return half ? C / 2 * upper + r * lower : r * upper; }
    // tokens of (half, sub), the 32 columns of f (not the right half of the upper rows)
    __device__ __forceinline__ void rows(int half, int sub, int f, bf16x8 (&o)[PLANES]) const
    {
        const __bf16 *p = at + line(half, row_of(0, sub)) + 32 * f + 8 * ((threadIdx.x & 63) >> 4);
#pragma unroll
        for (int i = 0; i < PLANES; ++i) o[i] = *reinterpret_cast<const bf16x8 *>(p + i * plane);
    }
    // columns of (f, sub), the 32 rows of `half`
    __device__ __forceinline__ void cols(int f, int sub, int half, bf16x8 (&o)[PLANES]) const
    {
        const int lane = threadIdx.x & 63, r = 8 * (lane >> 4) + ((lane & 15) >> 2);
        const __bf16 *p = at + line(half, r) + 32 * f + 8 * (lane & 3) + 4 * sub;
#pragma unroll
        for (int i = 0; i < PLANES; ++i) o[i] = transposed(p + i * plane, p + i * plane + 4 * (half ? lower : upper));
    }
};
// and its first PLANES terms on their way there, from where merit_delta_prepare leaves them
template <int PLANES, int THREADS> struct TriangleRows {
    static constexpr int per = TRIANGLE / 8, all = PLANES * per, units = (all + THREADS - 1) / THREADS;
    bf16x8 e[units];
    __device__ __forceinline__ void load(const __bf16 *from)
    {
#pragma unroll
        for (int i = 0; i < units; ++i) {
            const int u = (int)(threadIdx.x % THREADS) + i * THREADS;
            e[i] = reinterpret_cast<const bf16x8 *>(from)[u < all ? u : all - 1];
        }
    }
    __device__ __forceinline__ void store(const Triangle<PLANES> &t) const
    {
#pragma unroll
        for (int i = 0; i < units; ++i) {
            const int u = (int)(threadIdx.x % THREADS) + i * THREADS, v = u % per, w = v - per / 3;
            const int at = v < per / 3 ? t.line(0, v >> 2) + (v & 3) * 8 : t.line(1, w >> 3) + (w & 7) * 8;
            if (u < all) *reinterpret_cast<bf16x8 *>(t.at + u / per * t.plane + at) = e[i];
        }
    }
};
// What merit_delta_prepare leaves of a chunk of a head
struct Prepared {
    __bf16 *w, *mix;        // -W and P, three terms each
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

// Eight values of a row of n, from column c on.  Nothing stands in a branch, so that loads of many rows go out together, and what is read
// in the place of values that are not there is not looked at before `keep8` makes zeros of it, where the values are used: a select
// right behind a load waits for it.  WIDE: rows start on 16 bytes and n is a multiple of 8.
template <bool WIDE, typename T> __device__ __forceinline__ Eight<T> take8(const T *row, int c, int n)
{
    Eight<T> r;
    if constexpr (WIDE) {
        const u32x4 *from = reinterpret_cast<const u32x4 *>(row + (c < n ? c : 0));
        if constexpr (sizeof(T) == 2) {
            r.v = __builtin_bit_cast(typename Eight<T>::vec, from[0]);
        } else {
            const u32x4 a = from[0], b = from[1];
            r.v = __builtin_bit_cast(typename Eight<T>::vec, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = row[max(min(c + e, n - 1), 0)];       // (n may be 0: the row's first value is there)
    }
    return r;
}
template <bool WIDE, typename T> __device__ __forceinline__ Eight<T> keep8(const Eight<T> &x, int c, int n)
{
    Eight<T> r = zero8<T>();
    if constexpr (WIDE) {
        if (c < n) r = x;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < n) r.v[e] = x.v[e];
    }
    return r;
}

// A chunk's rows of q or k: unit u of a thread is row u / (KF * 4) of the tile and eight columns (with more threads than units some have
// the same).  FULL: all C rows are there, else m, at least one, the others zeros.
template <typename T, int KF, int THREADS> struct ChunkRows {
    static constexpr int all = C * KF * 4, units = (all + THREADS - 1) / THREADS, step = THREADS / (KF * 4);
    Eight<T> e[units];

    static __device__ __forceinline__ int unit() { return (int)(threadIdx.x % THREADS) % all; }
    template <bool FULL, bool WIDE>
    __device__ __forceinline__ void load(const Rows &x, int64_t b, int64_t t0, int m, int head, int D)
    {
        const int r0 = unit() / (KF * 4), c = unit() % (KF * 4) * 8;
        const T *from = static_cast<const T *>(x.data) + b * x.s0 + t0 * x.s1 + (int64_t)head * D;
        const T *row = from + r0 * x.s1;
#pragma unroll
        for (int i = 0; i < units; ++i) {
            if constexpr (FULL) {
                e[i] = take8<WIDE, T>(row + i * step * x.s1, c, D);
            } else {
                e[i] = take8<WIDE, T>(from + min(r0 + i * step, m - 1) * x.s1, c, D);
            }
        }
    }
    // (zeros in the place of what is not there)
    template <bool FULL, bool WIDE> __device__ __forceinline__ Eight<T> value(int i, int m, int D) const
    {
        const int r = unit() / (KF * 4) + i * step, c = unit() % (KF * 4) * 8;
        return keep8<WIDE, T>(e[i], c, FULL || r < m ? D : 0);
    }
    template <bool FULL, bool WIDE, typename M> __device__ __forceinline__ void store(const M &t, int m, int D) const
    {
#pragma unroll
        for (int i = 0; i < units; ++i) {
            bf16x8 o[Terms<T>::n];
            terms8<T>(value<FULL, WIDE>(i, m, D), o);
            t.put8(unit() / (KF * 4) + i * step, unit() % (KF * 4) * 8, o);
        }
    }
};

// A lane's values of a column of v or dy: N halves of a chunk from `half` on (each two results, sub 0 and 1, of four rows).  16-bit
// values stay as they were loaded, each in a register: putting two into one would wait for them.
template <typename T, int N> struct ChunkColumn {
    typedef typename std::conditional<sizeof(T) == 2, uint16_t, float>::type M;
    typedef typename std::conditional<sizeof(T) == 2, uint32_t, float>::type Word;
    Word v[2 * N][4];

    // `c`: a column that is there
    template <bool FULL> __device__ __forceinline__ void load(const Rows &x, int64_t b, int64_t t0, int half, int m, int64_t c)
    {
        const int r0 = 32 * half + 8 * ((threadIdx.x & 63) >> 4);
        const M *from = static_cast<const M *>(x.data) + b * x.s0 + t0 * x.s1 + c, *row = from + r0 * x.s1;
#pragma unroll
        for (int k = 0; k < 2 * N; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 32 * (k >> 1) + 4 * (k & 1) + r;
                if constexpr (FULL) {
                    v[k][r] = row[t * x.s1];
                } else {
                    const Word f = from[min(r0 + t, m - 1) * x.s1];
                    v[k][r] = r0 + t < m ? f : (Word)0;
                }
            }
    }
    __device__ __forceinline__ float value(int k, int r) const
    {
        if constexpr (sizeof(T) == 4) return v[k][r];
        else return (float)__builtin_bit_cast(T, (uint16_t)v[k][r]);
    }
};
// The results of half a chunk to a column of `x`: tokens from m on are zeros, those from `there` on are not
template <bool FULL, typename T>
__device__ __forceinline__ void put_column(const f32x4 (&v)[2], const Rows &x, int64_t b, int64_t t0, int half, int m, int there, int64_t c, bool in)
{
    const int r0 = 32 * half + 8 * ((threadIdx.x & 63) >> 4);
    T *row = static_cast<T *>(x.data) + b * x.s0 + (t0 + r0) * x.s1 + c;
    if (in)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = 4 * k + r;
                if (FULL || r0 + t < there) row[t * x.s1] = (T)(FULL || r0 + t < m ? v[k][r] : 0.0f);
            }
}
// 32 rows of fp32, of which `there` are there, to a column of rows of Dv; and back
__device__ __forceinline__ void put_rows(const f32x4 (&v)[2], float *out, int there, int64_t Dv, bool in)
{
    const int r0 = 8 * ((threadIdx.x & 63) >> 4);
    float *row = out + r0 * Dv;
    if (!in) return;
    if (there >= 32) {
#pragma unroll
        for (int t = 0; t < 8; ++t) row[t * Dv] = v[t >> 2][t & 3];
    } else {
#pragma unroll
        for (int t = 0; t < 8; ++t)
            if (r0 + t < there) row[t * Dv] = v[t >> 2][t & 3];
    }
}
__device__ __forceinline__ void get_rows(f32x4 (&v)[2], const float *from, int there, int64_t Dv, bool in)
{
    const int r0 = 8 * ((threadIdx.x & 63) >> 4);
#pragma unroll
    for (int t = 0; t < 8; ++t) v[t >> 2][t & 3] = from && in && r0 + t < there ? from[(r0 + t) * Dv] : 0.0f;
}

// What merit_delta_prepare leaves of a chunk of a head, 64 values each
enum { IN_K = 0,        // exp(G) / |k|
       BETA = 1,
       OUT_K = 2,       // exp(G_C - G) / |k|
       IN_Q = 3,        // scale exp(G) / |q|
       INV_K = 4, INV_Q = 5,                    // 1 / |k|, 1 / |q| (1 where they are taken as they are)
       SCALARS = 6 };
constexpr int SCALAR_FLOATS = DELTA_SCALAR_FLOATS;      // and G, to base 2 and in 64 bits, behind them
static_assert(SCALAR_FLOATS == SCALARS * C + 2 * C, "");

__device__ __forceinline__ int tokens_of(const DeltaParams &p, int64_t b)
{
    return p.lens ? min(max((int)p.lens[b], 0), (int)p.L) : (int)p.L;
}
// A decay's logarithm to base 2, in 64 bits.  (No decay of fp32 is below exp(-1000); -inf, which has no differences, included.)
__device__ __forceinline__ double log2_decay(float g) { return 1.44269504088896340736 * (g < -1000.0f ? -1000.0 : (double)g); }
// 2^x of a difference of sums of those.  The whole part goes into the exponent: rounded to fp32 with it, x would lose the digits that
// make the fraction's (44 x 2^-24 of 2^-86).
__device__ __forceinline__ float exp2_of(double x)
{
    const double whole = __builtin_rint(x);
    return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f((float)(x - whole)), (int)fmin(whole, 2000.0));
}

}  // namespace delta
}  // namespace merit
