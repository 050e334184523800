// The norms before and after a block, tensors of bfloat16 (one type a file: they compile side by side).
#include "block_norm.h"

namespace merit {
namespace block_norm {
hipError_t passes_bf16(const BlockNormParams &p, bool backward, hipStream_t s) { return passes<bf16_t>(p, backward, s); }
}  // namespace block_norm
}  // namespace merit
