// Shared by the plan code and the kernels of the operators along a sequence of tokens
// (include/merit_tokens.h).  Not part of the public ABI.
#pragma once

#include <stdint.h>
#include <hip/hip_runtime.h>

#include "merit_tokens.h"

namespace merit {

// ---- operands as the kernels see them ----------------------------------------
struct Rows {              // [d0, d1, dense...]: element (i, j) starts at data + i * s0 + j * s1 (elements)
    void *data;
    int64_t s0, s1;
};
struct Param {             // a dense vector or matrix of parameters: fp32 or the plan's type
    const void *data;
    int32_t f32;
};

// out[segment][j] = sum over r < rows of in[r * pitch + at + j], fp32: the last step of every sum over workgroups.  The rows
// go in a fixed order, so the result does not depend on which workgroup ended first.
struct ReduceSeg {
    float *out;            // nullptr: nobody wants it
    int64_t at, len;
};
struct ReduceParams {
    const float *in;
    int64_t rows, pitch;
    ReduceSeg seg[4];
    int nseg;
};
hipError_t launch_reduce_rows(const ReduceParams &p, hipStream_t s);

// ---- group norm ---------------------------------------------------------------
struct NormParams {
    int64_t N, S;
    int C, G, Cg;
    float eps;
    int act;
    int vec;               // channels a lane moves at once: 16 bytes of them, 8, 4 or one
    Rows x, y, dy, dx;
    Param w, b;
    float *mean, *rstd;    // [N, G]
    float *part;           // workspace
    int rows_form;         // one row a group
    int slab;              // a group a workgroup: its threads / 256 << 8 | units a thread (0: not this form)
    int ctiles;            // column tiles
    int group_tile;        // chunks: groups of a tile
    int64_t chunks;        // row chunks of an image; one row a group: workgroups along the rows
    int64_t chunk_rows;
    float *dw, *db;
};

// ---- causal convolution ----------------------------------------------------------
struct CconvParams {
    int64_t B, L;
    int D, K, act;
    int vec;
    Rows x, y, dy, dx, init, fin, dfin, dinit;
    Param w, b;
    const int32_t *lens;
    int strip;             // tokens a thread walks
    int64_t strips;        // of a sequence (at least 1)
    float *part;           // [row blocks][K + 1][D]
    int64_t row_blocks;
    float *dw, *db;
};

// ---- selective scan ----------------------------------------------------------------
struct ScanParams {
    int64_t B, L;
    int D, N, G, Dg;       // Dg = D / G channels share B and C
    int softplus;
    int type;              // merit_dtype of x, dt, B, C, z, y, ...
    uint32_t block0;       // workgroups of the launches before this one
    Rows x, dt, Bm, Cm, z, y, dy, dx, ddt, dz, dB, dC;
    const float *A, *skip, *dt_bias, *h0, *dh_last;
    const int32_t *lens;
    float *h_last, *states, *dh0;
    int64_t tiles;         // of MERIT_SCAN_TILE tokens
    int64_t chunk_tiles;   // tiles of a chunk (= tiles: one chunk)
    int chunks;
    int ctiles;            // channel tiles of a group
    float *chunk_h;        // [B, chunks, D, N]: what a chunk adds to the state (or to its adjoint)
    float *chunk_dt;       // [B, chunks, D]: its steps' sum
    float *part_bc;        // [G * ctiles][B, L][2][N]: dB, dC of a channel tile
    float *part_a;         // [B * chunks][D * N + 2 D]: dA, dskip, ddt_bias of a sequence's chunk
    float *dA, *dskip, *ddt_bias;
};
// lanes of a channel (scan.h: by_states)
constexpr int scan_lpc(int N) { return N == 1 ? 1 : N <= 8 ? 2 : N <= 16 ? 4 : N <= 32 ? 8 : 16; }
constexpr int SCAN_THREADS = 256;
// The forward pass has two halves of SCAN_THREADS in a workgroup, and a launch holds fewer than 2^32 threads: more workgroups go
// in launches of this many, one after the other.
constexpr int64_t SCAN_FORWARD_BLOCKS = (1ll << 32) / (2 * SCAN_THREADS) - 1;

}  // namespace merit

struct merit_token_plan {
    int kind;              // 0 norm, 1 convolution, 2 scan
    int type;              // merit_dtype
    merit::NormParams norm;
    merit::CconvParams conv;
    merit::ScanParams scan, scan_back;     // (in how many chunks: one choice for each direction)
};

namespace merit {
hipError_t launch_norm(const NormParams &p, int type, hipStream_t s);
hipError_t launch_norm_backward(const NormParams &p, int type, hipStream_t s);
hipError_t launch_cconv(const CconvParams &p, int type, hipStream_t s);
hipError_t launch_cconv_backward(const CconvParams &p, int type, hipStream_t s);
hipError_t launch_cconv_step(const CconvParams &p, int type, hipStream_t s);
hipError_t launch_scan(const ScanParams &p, hipStream_t s);
hipError_t launch_scan_backward(const ScanParams &p, hipStream_t s);
hipError_t launch_scan_step(const ScanParams &p, hipStream_t s);
}  // namespace merit

#ifdef __HIPCC__
namespace merit {

// ---- elements and vectors of them -------------------------------------------------
typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <typename T, int V> struct Vec { typedef T type __attribute__((ext_vector_type(V))); };
template <typename T> struct Vec<T, 1> { typedef T type; };
template <typename T, int V> using vec_t = typename Vec<T, V>::type;

template <typename T, int V> __device__ __forceinline__ float at(const vec_t<T, V> &v, int i)
{
    if constexpr (V == 1) return (float)v;
    else return (float)v[i];
}
template <typename T, int V> __device__ __forceinline__ void put(vec_t<T, V> &v, int i, float f)
{
    if constexpr (V == 1) v = (T)f;
    else v[i] = (T)f;
}
template <typename T, int V> __device__ __forceinline__ vec_t<T, V> load_vec(const void *base, int64_t at)
{
    return *reinterpret_cast<const vec_t<T, V> *>(static_cast<const T *>(base) + at);
}
template <typename T, int V> __device__ __forceinline__ void store_vec(void *base, int64_t at, const vec_t<T, V> &v)
{
    *reinterpret_cast<vec_t<T, V> *>(static_cast<T *>(base) + at) = v;
}
// COUNT parameters from element i on.  One branch for all of them: loads that each stand in a branch of their own are waited
// for one by one (16 of them were half of a norm's second launch).
template <typename T, int COUNT> __device__ __forceinline__ void load_params(Param p, int64_t i, float absent, float (&v)[COUNT])
{
    if (!p.data) {
#pragma unroll
        for (int k = 0; k < COUNT; ++k) v[k] = absent;
    } else if (p.f32) {
        const float *q = static_cast<const float *>(p.data) + i;
#pragma unroll
        for (int k = 0; k < COUNT; ++k) v[k] = q[k];
    } else {
        const T *q = static_cast<const T *>(p.data) + i;
#pragma unroll
        for (int k = 0; k < COUNT; ++k) v[k] = (float)q[k];
    }
}
template <typename T> __device__ __forceinline__ float load_param(Param p, int64_t i, float absent)
{
    float v[1];
    load_params<T>(p, i, absent, v);
    return v[0];
}

// ---- elementary functions -----------------------------------------------------------
constexpr float LOG2E = 1.44269504088896340736f;

__device__ __forceinline__ float sigmoidf(float u) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E * u)); }
__device__ __forceinline__ float siluf(float u) { return u * sigmoidf(u); }
// (SiLU of -inf is a NaN, -inf * 0, as the formula gives in any precision; a clipped NaN stays one)
__device__ __forceinline__ float apply_act(float u, int act)
{
    if (act == MERIT_ACT_SILU) return siluf(u);
    return act == MERIT_ACT_RELU ? (u > 0.0f || u != u ? u : 0.0f) : u;
}
__device__ __forceinline__ float act_slope(float u, int act)
{
    if (act == MERIT_ACT_SILU) {
        const float q = sigmoidf(u);
        return q * (1.0f + u * (1.0f - q));
    }
    return act == MERIT_ACT_RELU ? (u > 0.0f ? 1.0f : 0.0f) : 1.0f;
}

// ---- sums over lanes ------------------------------------------------------------------
// v + (v of the lane whose number differs in bit BIT)
template <int BIT> __device__ __forceinline__ float lane_xor(float v)
{
    const int i = __builtin_bit_cast(int, v);
    int o;
    if constexpr (BIT == 0) o = __builtin_amdgcn_mov_dpp(i, 0xB1, 0xF, 0xF, true);            // quad_perm 1,0,3,2
    else if constexpr (BIT == 1) o = __builtin_amdgcn_mov_dpp(i, 0x4E, 0xF, 0xF, true);       // quad_perm 2,3,0,1
    else if constexpr (BIT == 2) o = __builtin_amdgcn_ds_swizzle(i, 0x1F | (4 << 10));
    else if constexpr (BIT == 3) o = __builtin_amdgcn_mov_dpp(i, 0x128, 0xF, 0xF, true);      // row_ror:8
    else if constexpr (BIT == 4) o = __builtin_amdgcn_ds_swizzle(i, 0x1F | (16 << 10));
    else o = __shfl_xor(i, 32);
    return __builtin_bit_cast(float, o);
}
// the sum over aligned runs of `lanes` (a power of two) lanes, in every one of them
__device__ __forceinline__ float sum_lanes(float v, int lanes)
{
    if (lanes > 1) v += lane_xor<0>(v);
    if (lanes > 2) v += lane_xor<1>(v);
    if (lanes > 4) v += lane_xor<2>(v);
    if (lanes > 8) v += lane_xor<3>(v);
    if (lanes > 16) v += lane_xor<4>(v);
    if (lanes > 32) v += lane_xor<5>(v);
    return v;
}

}  // namespace merit
#endif
