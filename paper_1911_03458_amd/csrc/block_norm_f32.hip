// The norms before and after a block, tensors of fp32 (one type a file: they compile side by side).
#include "block_norm.h"

namespace merit {
namespace block_norm {
hipError_t passes_f32(const BlockNormParams &p, bool backward, hipStream_t s) { return passes<float>(p, backward, s); }
}  // namespace block_norm
}  // namespace merit

namespace merit {

namespace {
hipError_t any_type(const BlockNormParams &p, bool backward, hipStream_t s)
{
    if (p.type == MERIT_F32) return block_norm::passes_f32(p, backward, s);
    return p.type == MERIT_F16 ? block_norm::passes_f16(p, backward, s) : block_norm::passes_bf16(p, backward, s);
}
}  // namespace

hipError_t launch_block_norm(const BlockNormParams &p, hipStream_t s) { return any_type(p, false, s); }

hipError_t launch_block_norm_backward(const BlockNormParams &p, hipStream_t s)
{
    if (hipError_t e = any_type(p, true, s)) return e;
    ReduceParams r = {};
    r.in = p.part;
    r.rows = p.blocks;
    r.pitch = 5ll * p.C;
    float *const want[5] = {p.daw, p.dab, p.dscale, p.dbw, p.dbb};
    for (int k = 0; k < 5; ++k)
        if (want[k]) r.seg[r.nseg++] = {want[k], (int64_t)k * p.C, p.C};
    return r.nseg ? launch_reduce_rows(r, s) : hipSuccess;
}

}  // namespace merit
