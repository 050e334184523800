// The gated delta rule on tensors of bfloat16 (one type a file: they compile side by side).
#include "delta_backward.h"

namespace merit {
namespace delta {
hipError_t passes_bf16(const DeltaParams &p, int pass, hipStream_t s) { return passes<bf16_t>(p, pass, s); }
}  // namespace delta

}  // namespace merit
