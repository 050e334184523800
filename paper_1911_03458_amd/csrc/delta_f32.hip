// The gated delta rule on tensors of fp32 (one type a file: they compile side by side).
#include "delta_backward.h"

namespace merit {
namespace delta {
hipError_t passes_f32(const DeltaParams &p, int pass, hipStream_t s) { return passes<float>(p, pass, s); }
}  // namespace delta

namespace {
hipError_t any_type(const DeltaParams &p, int pass, hipStream_t s)
{
    if (p.type == MERIT_F32) return delta::passes_f32(p, pass, s);
    return p.type == MERIT_F16 ? delta::passes_f16(p, pass, s) : delta::passes_bf16(p, pass, s);
}
}  // namespace

hipError_t launch_delta(const DeltaParams &p, hipStream_t s) { return any_type(p, delta::FORWARD, s); }
hipError_t launch_delta_backward(const DeltaParams &p, hipStream_t s) { return any_type(p, delta::BACKWARD, s); }
hipError_t launch_delta_step(const DeltaParams &p, hipStream_t s) { return any_type(p, delta::STEP, s); }

}  // namespace merit
