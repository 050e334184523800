// The norms before and after a block, tensors of binary16 (one type a file: they compile side by side).
#include "block_norm.h"

namespace merit {
namespace block_norm {
hipError_t passes_f16(const BlockNormParams &p, bool backward, hipStream_t s) { return passes<f16_t>(p, backward, s); }
}  // namespace block_norm
}  // namespace merit
