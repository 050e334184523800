// Device helpers of the gated delta rule's kernels (delta.hip, delta_backward.hip).
//
//     S_t = a_t S_{t-1} + k_t u_t^T,   u_t = b_t d_t,   d_t = v_t - a_t S_{t-1}^T k_t,   y_t = scale S_t^T q_t,   a_t = exp(g_t)
//
// A chunk of C = 64 tokens at once, G_t = g_1 + .. + g_t inside it, f_tj = exp(G_t - G_j), N_tj = f_tj k_t.k_j below the diagonal:
//     d = (1 + N diag(b))^-1 (v - exp(G) K S_0),    y = scale (exp(G) Q S_0 + (f o Q K^T) u),    S_C = exp(G_C) S_0 + K^T (exp(G_C - G) u)
// so that a token's dependence on those before it is a triangular matrix (found by merit_delta_prepare for all chunks side by
// side), and the rest are matrix products.
//
// Products run on v_mfma_f32_16x16x32_bf16.  An fp32 operand goes in as three bfloat16 terms of 8 bits each (x = x0 + x1 + x2 with
// the rounding error of the one before in each), a binary16 one as two, a bfloat16 one as it is, and terms whose product is below
// 2^-24 of the leading one are left out: 3 products for an exact operand with an fp32 one, 6 for two fp32 ones, at a sixteenth of
// the time each that v_mfma_f32_16x16x4_f32 takes.  States, sums and what is kept of them are fp32.
#pragma once

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

// Terms of P and u where they give y, which is rounded to T: two leave 2^-17, next to the 2^-12 of a rounding to binary16; the
// gradients that P gives go on into sums in fp32
template <typename T> constexpr int mix_terms(bool backward) { return backward || Terms<T>::n == 3 ? 3 : 2; }

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

// ---- operands -----------------------------------------------------------------------------------------------
// Eight values of a row from column c on, zeros from column n on.  wide: rows start on 16 bytes and n is a multiple of 8.
template <typename T> struct Eight { T v[8]; };
template <typename T> __device__ __forceinline__ Eight<T> load8(const T *row, int c, int n, bool wide)
{
    Eight<T> r;
    if (wide) {
        typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
        u32x4_t raw[sizeof(T) / 2];
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) raw[i] = u32x4_t{0, 0, 0, 0};
        if (c < n)
#pragma unroll
            for (int i = 0; i < (int)(sizeof(T) / 2); ++i) raw[i] = reinterpret_cast<const u32x4_t *>(row + c)[i];
        __builtin_memcpy(&r, raw, sizeof(r));
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = c + e < n ? row[c + e] : (T)0.0f;
    }
    return r;
}
template <typename T> __device__ __forceinline__ Eight<T> zero8()
{
    Eight<T> r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = (T)0.0f;
    return r;
}
template <typename T> __device__ __forceinline__ void terms8(const Eight<T> &x, bf16x8 (&o)[Terms<T>::n])
{
    if constexpr (Terms<T>::n == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[0][e] = x.v[e];
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

// A chunk's rows of q or k: unit u of a thread is row u / (KF * 4) of the tile and eight columns
template <typename T, int KF> struct ChunkRows {
    static constexpr int units = C * KF * 4 / NT;
    Eight<T> e[units];

    __device__ __forceinline__ void load(const Rows &x, int64_t b, int64_t t0, int m, int head, int D, bool wide)
    {
#pragma unroll
        for (int i = 0; i < units; ++i) {
            const int u = (int)threadIdx.x + i * NT, r = u / (KF * 4), c = u % (KF * 4) * 8;
            e[i] = zero8<T>();
            if (r < m)
                e[i] = load8<T>(static_cast<const T *>(x.data) + b * x.s0 + (t0 + r) * x.s1 + (int64_t)head * D, c, D, wide);
        }
    }
    __device__ __forceinline__ void store(const Tile<Terms<T>::n, C, KF * 32> &t) const
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
