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
    int64_t b;             // sequence
    int n;                 // its tokens
    int chunk, g, ct;
    int d, lane;           // channel (of a lane that has none: the group's last), the lane's number among its channel's
    bool in;               // the channel is there
    int tile0, tile1;      // tiles of the chunk
    int tend;              // the first of them that has no token of the sequence
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
    w.d = w.g * p.Dg + min(cl, p.Dg - 1);
    w.n = p.lens ? min(max(p.lens[w.b], 0), (int)p.L) : (int)p.L;
    w.tile0 = w.chunk * (int)p.chunk_tiles;
    w.tile1 = min(w.tile0 + (int)p.chunk_tiles, (int)p.tiles);
    w.tend = min(w.tile1, (w.n + TT - 1) / TT);
    return w;
}

// Loads go out without a branch and stay raw (a 16-bit element in the low half) until their values are wanted, a tile later:
// a guarded load would be waited for where the guard ends.  Tokens behind the end, channels and states that are not there
// read the last one that is, and are replaced by zeros when the values are made.  Not called for a sequence of no tokens.
template <int COUNT, typename F>
__device__ __forceinline__ void load_raw(const void *base, int type, uint32_t (&v)[COUNT], F &&at)
{
    if (type == MERIT_F32) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = static_cast<const uint32_t *>(base)[at(i)];
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = static_cast<const uint16_t *>(base)[at(i)];
    }
}
template <int COUNT> __device__ __forceinline__ void values(const uint32_t (&raw)[COUNT], int type, float (&v)[COUNT])
{
    if (type == MERIT_BF16) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = __builtin_bit_cast(float, raw[i] << 16);
    } else if (type == MERIT_F16) {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = (float)__builtin_bit_cast(f16_t, (uint16_t)raw[i]);
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = __builtin_bit_cast(float, raw[i]);
    }
}

// the lane's tokens of a tile, in the channel
template <int SPL, int LPC>
__device__ __forceinline__ void load_rows(const Rows &r, int type, const Where &w, int tile, uint32_t (&v)[Shape<SPL, LPC>::TPL])
{
    load_raw(r.data, type, v, [&](int i) { return w.b * r.s0 + min(tile * TT + i * LPC + w.lane, w.n - 1) * r.s1 + w.d; });
}
// the thread's elements of B or C of a tile
template <int SPL, int LPC>
__device__ __forceinline__ void load_states(const Rows &r, const ScanParams &p, const Where &w, int tile, uint32_t (&v)[Shape<SPL, LPC>::EB])
{
    constexpr int NP = Shape<SPL, LPC>::NP;
    load_raw(r.data, p.type, v, [&](int i) {
        const int e = (i * NT + (int)threadIdx.x) & (TT * NP - 1), n = e % NP;
        return w.b * r.s0 + min(tile * TT + e / NP, w.n - 1) * r.s1 + w.g * p.N + min(n, p.N - 1);
    });
}
template <int SPL, int LPC>
__device__ __forceinline__ void stage_states(float *lds, const ScanParams &p, const Where &w, int tile, const uint32_t (&raw)[Shape<SPL, LPC>::EB])
{
    constexpr int NP = Shape<SPL, LPC>::NP;
    float v[Shape<SPL, LPC>::EB];
    values(raw, p.type, v);
#pragma unroll
    for (int i = 0; i < Shape<SPL, LPC>::EB; ++i) {
        const int e = i * NT + (int)threadIdx.x;
        if (e < TT * NP) lds[e] = e % NP < p.N && tile * TT + e / NP < w.n ? v[i] : 0.0f;
    }
}

// A barrier for LDS alone: loads from memory stay in flight across it
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
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
