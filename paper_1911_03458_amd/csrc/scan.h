// What the scan's kernels share (scan.hip: forward and single tokens, scan_backward.hip).
#pragma once
#include <type_traits>

#include "tokens.h"

namespace merit {
namespace scan {

constexpr int TT = MERIT_SCAN_TILE, NT = SCAN_THREADS;

// LPC lanes have a channel, SPL states each.  PAD: N < SPL LPC, the states behind N stay 0.
template <int SPL, int LPC> struct Shape {
    static constexpr int NP = SPL * LPC;           // states, padded
    static constexpr int CPB = NT / LPC;           // channels of a workgroup
    // Of a tile's tokens a channel's lanes load every LQ-th, lane j tokens j, j + LQ, ...; eight and sixteen lanes do as
    // two and four quads that load the same, since a value reaches the lanes of its quad inside the instruction that uses
    // it and lanes beyond it only by way of LDS.
    static constexpr int LQ = LPC < 4 ? LPC : 4;
    static constexpr int TPL = TT / LQ;
    static constexpr int EB = (TT * NP + NT - 1) / NT;     // elements of B (and of C) of a tile that a thread stages
};

struct Where {
    int64_t b;             // sequence
    int n;                 // its tokens
    int chunk, g, ct;
    int d, lane;           // channel (of a lane that has none: the group's last), the lane's number among its channel's
    int tok;               // the first of its tokens in a tile
    bool in;               // the channel is there
    int tile0, tile1;      // tiles of the chunk
    int tend;              // the first of them that has no token of the sequence
};
// The workgroup's part: `chunks` chunks of every sequence, from `first` on
template <int LPC> __device__ __forceinline__ Where where(const ScanParams &p, int first, int chunks, int thread)
{
    Where w;
    uint32_t r = p.block0 + blockIdx.x;
    w.ct = (int)(r % (uint32_t)p.ctiles);
    r /= (uint32_t)p.ctiles;
    w.g = (int)(r % (uint32_t)p.G);
    r /= (uint32_t)p.G;
    w.chunk = first + (int)(r % (uint32_t)chunks);
    w.b = r / (uint32_t)chunks;
    const int cl = w.ct * (NT / LPC) + thread / LPC;
    w.lane = thread & (LPC - 1);
    w.tok = w.lane & 3;
    w.in = cl < p.Dg;
    w.d = w.g * p.Dg + min(cl, p.Dg - 1);
    w.n = p.lens ? min(max(p.lens[w.b], 0), (int)p.L) : (int)p.L;
    w.tile0 = w.chunk * (int)p.chunk_tiles;
    w.tile1 = min(w.tile0 + (int)p.chunk_tiles, (int)p.tiles);
    w.tend = min(w.tile1, (w.n + TT - 1) / TT);
    return w;
}

// How the kernels move tiles.  Loads go out two tiles before their use (backward one) and stay raw (a 16-bit element in the low half) until
// then.  Loads and stores share one counter and the wait for a load waits for what was issued before it, so a tile's results
// are written while the next tile is under way, before its own loads are issued: a store is never younger than a load that
// is waited for.  The barrier between staging and reading LDS waits for LDS alone (lds_barrier).
// (Results written at once and a barrier that waits for everything took a forward pass from 263 to 373 us.)
// A tensor as a lane walks it: the address (in global memory: a flat load would count as one from LDS too) of its first
// element of tile 0, bytes from token to token.
typedef __attribute__((address_space(1))) char *gptr;
struct Walk {
    gptr at;
    int64_t step;
};
template <typename T> using raw_t = std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t>;
template <typename T> __device__ __forceinline__ Walk walk_rows(const Rows &r, const Where &w)
{
    constexpr int64_t es = sizeof(T);
    return Walk{(gptr)r.data + (w.b * r.s0 + w.tok * r.s1 + w.d) * es, r.s1 * es};
}
// (thread e of a tile's TT x NP elements of B or C, further ones NT elements on)
template <typename T, int NP> __device__ __forceinline__ Walk walk_states(const Rows &r, const ScanParams &p, const Where &w, int thread)
{
    constexpr int64_t es = sizeof(T);
    const int e = thread & (TT * NP - 1);
    return Walk{(gptr)r.data + (w.b * r.s0 + (e / NP) * r.s1 + w.g * p.N + min(e % NP, p.N - 1)) * es, r.s1 * es};
}
// COUNT elements, `every` tokens apart, the first token `first` of tile `tile`.  WHOLE: all of the tile's tokens are there
// and the addresses differ from the lane's by numbers that all lanes share (a product of 64 bits a load and lane costs more
// than the scan's arithmetic); else tokens behind `last` read that one again.
template <typename T, bool WHOLE, int COUNT>
__device__ __forceinline__ void load_walk(const Walk &k, int tile, int every, int first, int last, raw_t<T> (&v)[COUNT])
{
    const int64_t off = (int64_t)(tile * TT) * k.step;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const gptr at = WHOLE ? k.at + (off + (int64_t)(i * every) * k.step)
                              : k.at + (int64_t)(min(tile * TT + i * every + first, last) - first) * k.step;
        v[i] = *reinterpret_cast<__attribute__((address_space(1))) const raw_t<T> *>(at);
    }
}
// ALL: every token of the tile is there; else only tokens before `end` are written
template <typename T, bool ALL, int COUNT>
__device__ __forceinline__ void store_walk(const Walk &k, int tile, int every, int first, int64_t end, const float (&v)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i)
        if (ALL || tile * TT + i * every + first < end)
            *reinterpret_cast<__attribute__((address_space(1))) T *>(k.at + (int64_t)(tile * TT + i * every) * k.step) = (T)v[i];
}
template <typename T, int COUNT> __device__ __forceinline__ void values(const raw_t<T> (&raw)[COUNT], float (&v)[COUNT])
{
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        if constexpr (std::is_same_v<T, bf16_t>) v[i] = __builtin_bit_cast(float, (uint32_t)raw[i] << 16);
        else v[i] = (float)__builtin_bit_cast(T, raw[i]);
    }
}

template <typename T, int SPL, int LPC>
__device__ __forceinline__ void stage_states(float *lds, const ScanParams &p, const Where &w, int thread, int tile, const raw_t<T> (&raw)[Shape<SPL, LPC>::EB])
{
    constexpr int NP = Shape<SPL, LPC>::NP;
    float v[Shape<SPL, LPC>::EB];
    values<T>(raw, v);
#pragma unroll
    for (int i = 0; i < Shape<SPL, LPC>::EB; ++i) {
        const int e = i * NT + thread;
        if (e < TT * NP) lds[e] = e % NP < p.N && tile * TT + e / NP < w.n ? v[i] : 0.0f;
    }
}

// A barrier for LDS alone: loads from memory stay in flight across it, which a fence would wait for
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// log(1 + exp(v)) = max(v, 0) + log1p(e), e = exp(-|v|); log1p(e) = log(u) + (e - (u - 1)) / u, u the rounded 1 + e, which
// gives back the digits of a small e that the sum cuts off
__device__ __forceinline__ float softplusf(float v)
{
    const float e = __builtin_amdgcn_exp2f(-LOG2E * __builtin_fabsf(v)), u = 1.0f + e;
    const float lost = e - (u - 1.0f);
    return fmaxf(v, 0.0f) + fmaf(__builtin_amdgcn_logf(u), 1.0f / LOG2E, lost * __builtin_amdgcn_rcpf(u));
}

#define MERIT_DPP(v, ctrl) __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), ctrl, 0xF, 0xF, true))
// the value that lane `j` of the lane's LQ has
template <int LQ> __device__ __forceinline__ float from_lane(float v, int j)
{
    if constexpr (LQ == 1) return v;
    else if constexpr (LQ == 2) return j ? MERIT_DPP(v, 0xF5) : MERIT_DPP(v, 0xA0);       // quad_perm 1,1,3,3 / 0,0,2,2
    else switch (j) {
    case 0: return MERIT_DPP(v, 0x00);
    case 1: return MERIT_DPP(v, 0x55);
    case 2: return MERIT_DPP(v, 0xAA);
    default: return MERIT_DPP(v, 0xFF);
    }
}

// the sum over the channel's lanes, in all of them
template <int LPC> __device__ __forceinline__ float sum_channel(float v)
{
    if constexpr (LPC > 8) v += MERIT_DPP(v, 0x140);       // row_mirror: the other eight of sixteen
    if constexpr (LPC > 4) v += MERIT_DPP(v, 0x141);       // row_half_mirror: the other quad of eight
    if constexpr (LPC > 1) v += MERIT_DPP(v, 0xB1);
    if constexpr (LPC > 2) v += MERIT_DPP(v, 0x4E);
    return v;
}

// v[u] of four tokens summed over the channel's lanes, each into the lane that has the token: out[0 .. 4 / LQ - 1].  A
// lane adds what it keeps to what its neighbour gives away, so a sum of four tokens takes three exchanges, not eight.
template <int LPC> __device__ __forceinline__ void sum_to_tokens(const float (&v)[4], float *out)
{
    if constexpr (LPC == 1) {
#pragma unroll
        for (int u = 0; u < 4; ++u) out[u] = v[u];
    } else {
        float q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            q[u] = v[u];
            if constexpr (LPC > 8) q[u] += MERIT_DPP(q[u], 0x140);
            if constexpr (LPC > 4) q[u] += MERIT_DPP(q[u], 0x141);
        }
        const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
        const float a = odd ? q[1] : q[0], ga = odd ? q[0] : q[1], b = odd ? q[3] : q[2], gb = odd ? q[2] : q[3];
        const float ra = a + MERIT_DPP(ga, 0xB1), rb = b + MERIT_DPP(gb, 0xB1);
        if constexpr (LPC == 2) {
            out[0] = ra;
            out[1] = rb;
        } else {
            const float keep = high ? rb : ra, give = high ? ra : rb;
            out[0] = keep + MERIT_DPP(give, 0x4E);
        }
    }
}

// one, two or four consecutive floats of LDS
template <int SPL> __device__ __forceinline__ void read_states(const float *at, float (&v)[SPL])
{
    if constexpr (SPL == 4) {
        const float4 q = *reinterpret_cast<const float4 *>(at);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else if constexpr (SPL == 2) {
        const float2 q = *reinterpret_cast<const float2 *>(at);
        v[0] = q.x, v[1] = q.y;
    } else v[0] = at[0];
}

template <int SPL> __device__ __forceinline__ void write_states(float *at, const float (&v)[SPL])
{
    if constexpr (SPL == 4) *reinterpret_cast<float4 *>(at) = make_float4(v[0], v[1], v[2], v[3]);
    else if constexpr (SPL == 2) *reinterpret_cast<float2 *>(at) = make_float2(v[0], v[1]);
    else at[0] = v[0];
}

// the same to memory, where a state need not start on more than its own boundary
template <int SPL> __device__ __forceinline__ void store_states(float *at, const float (&v)[SPL])
{
    typedef float vec __attribute__((ext_vector_type(SPL == 1 ? 2 : SPL), aligned(4)));
    if constexpr (SPL == 1) at[0] = v[0];
    else {
        vec q;
#pragma unroll
        for (int s = 0; s < SPL; ++s) q[s] = v[s];
        *reinterpret_cast<vec *>(at) = q;
    }
}

// A state (or its adjoint) through `count` chunks from `q` on: their decay, then what they add.  Four chunks' loads go out
// together.  No decay is 0: an infinite state stays one where fp32 cannot hold a chunk's.
template <int SPL>
__device__ __forceinline__ void through_chunks(const ScanParams &p, const Where &w, int n0, const float (&A2)[SPL], const bool (&ok)[SPL],
                                               float (&h)[SPL], int q, int count, int dir)
{
    constexpr int AT_ONCE = 4;
    for (; count > 0; count -= AT_ONCE, q += dir * AT_ONCE) {
        float sum[AT_ONCE], add[AT_ONCE][SPL];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int64_t at = (w.b * p.chunks + q + dir * min(k, count - 1)) * p.D + w.d;
            sum[k] = p.chunk_dt[at];
#pragma unroll
            for (int s = 0; s < SPL; ++s) add[k][s] = p.chunk_h[at * p.N + min(n0 + s, p.N - 1)];
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k)
            if (k < count)
#pragma unroll
                for (int s = 0; s < SPL; ++s)
                    if (ok[s]) {
                        const float decay = __builtin_amdgcn_exp2f(sum[k] * A2[s]);
                        h[s] = fmaf(decay == 0.0f && __builtin_isinf(h[s]) ? 1.0f : decay, h[s], add[k][s]);
                    }
    }
}

// a launch for the plan's number of states: F::run<SPL, LPC, PAD>()
template <typename F> hipError_t by_states(int N, F &&f)
{
    if (N == 1) return f.template run<1, 1, false>();
    if (N == 2) return f.template run<1, 2, false>();
    if (N == 4) return f.template run<2, 2, false>();
    if (N < 4) return f.template run<2, 2, true>();
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

// one of these per element type, each in a source of its own (they take long to compile)
template <typename T> hipError_t scan_backward_of(const ScanParams &p, hipStream_t s);

}  // namespace merit
