// The gated delta rule on tensors of binary16 (one type a file: they compile side by side).
#include "delta_backward.h"

namespace merit {
namespace delta {
hipError_t passes_f16(const DeltaParams &p, int pass, hipStream_t s) { return passes<f16_t>(p, pass, s); }
}  // namespace delta

}  // namespace merit
