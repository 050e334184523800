// What the scan's kernels share (scan.hip: forward and single tokens, scan_backward.hip).
#pragma once
#include "tokens.h"

namespace merit {
namespace scan {

constexpr int TT = MERIT_SCAN_TILE, NT = SCAN_THREADS;

// LPC lanes have a channel, SPL states each.  PAD: N < SPL LPC, the states behind N stay 0.
template <int SPL, int LPC> struct Shape {
    static constexpr int NP = SPL * LPC;           // states, padded
    static constexpr int CPB = NT / LPC;           // channels of a workgroup
    static constexpr int TPL = TT / LPC;           // tokens of a tile whose inputs a lane loads: j, j + LPC, ...
    static constexpr int EB = (TT * NP + NT - 1) / NT;     // elements of B (and of C) of a tile that a thread stages
};

struct Where {
    int64_t b, n;          // sequence, its tokens
    int chunk, g, ct;
    int d, lane;           // channel, the lane's number among its channel's
    bool in;               // the channel is there
    int64_t tile0, tile1;  // tiles of the chunk
};
template <int LPC> __device__ __forceinline__ Where where(const ScanParams &p, int chunks)
{
    Where w;
    uint32_t r = blockIdx.x;
    w.ct = (int)(r % (uint32_t)p.ctiles);
    r /= (uint32_t)p.ctiles;
    w.g = (int)(r % (uint32_t)p.G);
    r /= (uint32_t)p.G;
    w.chunk = (int)(r % (uint32_t)chunks);
    w.b = r / (uint32_t)chunks;
    const int cl = w.ct * (NT / LPC) + (int)threadIdx.x / LPC;
    w.lane = (int)threadIdx.x & (LPC - 1);
    w.in = cl < p.Dg;
    w.d = w.g * p.Dg + cl;
    w.n = p.lens ? min((int64_t)max(p.lens[w.b], 0), p.L) : p.L;
    w.tile0 = w.chunk * p.chunk_tiles;
    w.tile1 = min(w.tile0 + p.chunk_tiles, p.tiles);
    return w;
}

// The tokens of tile `tile` that belong to the lane, 0 behind the sequence's end
template <typename T, int SPL, int LPC>
__device__ __forceinline__ void load_rows_t(const Rows &r, const Where &w, int64_t tile, float (&v)[Shape<SPL, LPC>::TPL])
{
    const T *base = static_cast<const T *>(r.data) + w.b * r.s0 + w.d;
#pragma unroll
    for (int i = 0; i < Shape<SPL, LPC>::TPL; ++i) {
        const int64_t t = tile * TT + i * LPC + w.lane;
        v[i] = w.in && t < w.n ? (float)base[t * r.s1] : 0.0f;
    }
}
template <int SPL, int LPC>
__device__ __forceinline__ void load_rows(const Rows &r, int type, const Where &w, int64_t tile, float (&v)[Shape<SPL, LPC>::TPL])
{
    if (type == MERIT_BF16) load_rows_t<bf16_t, SPL, LPC>(r, w, tile, v);
    else if (type == MERIT_F16) load_rows_t<f16_t, SPL, LPC>(r, w, tile, v);
    else load_rows_t<float, SPL, LPC>(r, w, tile, v);
}

// The thread's elements of B or C of a tile, 0 behind the end and behind N
template <typename T, int SPL, int LPC>
__device__ __forceinline__ void load_states_t(const Rows &r, const ScanParams &p, const Where &w, int64_t tile,
                                              float (&v)[Shape<SPL, LPC>::EB])
{
    constexpr int NP = Shape<SPL, LPC>::NP;
    const T *base = static_cast<const T *>(r.data) + w.b * r.s0 + (int64_t)w.g * p.N;
#pragma unroll
    for (int i = 0; i < Shape<SPL, LPC>::EB; ++i) {
        const int e = i * NT + (int)threadIdx.x, n = e % NP;
        const int64_t t = tile * TT + e / NP;
        v[i] = e < TT * NP && n < p.N && t < w.n ? (float)base[t * r.s1 + n] : 0.0f;
    }
}
template <int SPL, int LPC>
__device__ __forceinline__ void load_states(const Rows &r, const ScanParams &p, const Where &w, int64_t tile,
                                            float (&v)[Shape<SPL, LPC>::EB])
{
    if (p.type == MERIT_BF16) load_states_t<bf16_t, SPL, LPC>(r, p, w, tile, v);
    else if (p.type == MERIT_F16) load_states_t<f16_t, SPL, LPC>(r, p, w, tile, v);
    else load_states_t<float, SPL, LPC>(r, p, w, tile, v);
}
template <int SPL, int LPC>
__device__ __forceinline__ void stage_states(float *lds, const float (&v)[Shape<SPL, LPC>::EB])
{
#pragma unroll
    for (int i = 0; i < Shape<SPL, LPC>::EB; ++i) {
        const int e = i * NT + (int)threadIdx.x;
        if (e < TT * Shape<SPL, LPC>::NP) lds[e] = v[i];
    }
}

__device__ __forceinline__ void store_el(void *base, int type, int64_t at, float v)
{
    if (type == MERIT_BF16) static_cast<bf16_t *>(base)[at] = (bf16_t)v;
    else if (type == MERIT_F16) static_cast<f16_t *>(base)[at] = (f16_t)v;
    else static_cast<float *>(base)[at] = v;
}
__device__ __forceinline__ float load_el(const void *base, int type, int64_t at)
{
    if (type == MERIT_BF16) return (float)static_cast<const bf16_t *>(base)[at];
    if (type == MERIT_F16) return (float)static_cast<const f16_t *>(base)[at];
    return static_cast<const float *>(base)[at];
}

// log(1 + exp(v)) = max(v, 0) + log1p(exp(-|v|)); log1p by log(1 + e) e / ((1 + e) - 1), which keeps the digits of a
// small e that the sum cuts off
__device__ __forceinline__ float softplusf(float v)
{
    const float e = __builtin_amdgcn_exp2f(-LOG2E * __builtin_fabsf(v)), u = 1.0f + e, d = u - 1.0f;
    const float l = d > 0.0f ? __builtin_amdgcn_logf(u) * (1.0f / LOG2E) * (e * __builtin_amdgcn_rcpf(d)) : e;
    return v != v ? v : fmaxf(v, 0.0f) + l;
}

// the value that lane `j` of the channel's lanes has
template <int LPC> __device__ __forceinline__ float from_lane(float v, int j);
template <> __device__ __forceinline__ float from_lane<1>(float v, int) { return v; }
#define MERIT_DPP(v, ctrl) __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), ctrl, 0xF, 0xF, true))
template <> __device__ __forceinline__ float from_lane<2>(float v, int j)
{
    return j ? MERIT_DPP(v, 0xF5) : MERIT_DPP(v, 0xA0);                 // quad_perm 1,1,3,3 / 0,0,2,2
}
template <> __device__ __forceinline__ float from_lane<4>(float v, int j)
{
    switch (j) {
    case 0: return MERIT_DPP(v, 0x00);
    case 1: return MERIT_DPP(v, 0x55);
    case 2: return MERIT_DPP(v, 0xAA);
    default: return MERIT_DPP(v, 0xFF);
    }
}
template <> __device__ __forceinline__ float from_lane<8>(float v, int j)
{
    return __shfl(v, ((int)threadIdx.x & 56) | j);
}
template <> __device__ __forceinline__ float from_lane<16>(float v, int j)
{
    return __shfl(v, ((int)threadIdx.x & 48) | j);
}

// the sum over the channel's lanes, in all of them
template <int LPC> __device__ __forceinline__ float sum_channel(float v)
{
    if constexpr (LPC > 1) v += MERIT_DPP(v, 0xB1);
    if constexpr (LPC > 2) v += MERIT_DPP(v, 0x4E);
    if constexpr (LPC > 4) v += MERIT_DPP(v, 0x141);       // row_half_mirror: the other quad of eight lanes
    if constexpr (LPC > 8) v += MERIT_DPP(v, 0x140);       // row_mirror: the other eight of sixteen
    return v;
}

// four consecutive floats of LDS or one
template <int SPL> __device__ __forceinline__ void read_states(const float *at, float (&v)[SPL])
{
    if constexpr (SPL == 4) {
        const float4 q = *reinterpret_cast<const float4 *>(at);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
#pragma unroll
        for (int s = 0; s < SPL; ++s) v[s] = at[s];
    }
}

// a launch for the plan's number of states: F::run<SPL, LPC, PAD>()
template <typename F> hipError_t by_states(int N, F &&f)
{
    if (N == 1) return f.template run<1, 1, false>();
    if (N == 4) return f.template run<4, 1, false>();
    if (N < 4) return f.template run<4, 1, true>();
    if (N == 8) return f.template run<4, 2, false>();
    if (N < 8) return f.template run<4, 2, true>();
    if (N == 16) return f.template run<4, 4, false>();
    if (N < 16) return f.template run<4, 4, true>();
    if (N == 32) return f.template run<4, 8, false>();
    if (N < 32) return f.template run<4, 8, true>();
    if (N == 64) return f.template run<4, 16, false>();
    return f.template run<4, 16, true>();
}

}  // namespace scan
}  // namespace merit
