// The scan's backward pass on bfloat16 tensors (scan_backward.h).
#include "scan_backward.h"

namespace merit {

template hipError_t scan_backward_of<bf16_t>(const ScanParams &p, hipStream_t s);

}  // namespace merit
