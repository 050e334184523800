// The scan's backward pass on fp32 tensors (scan_backward.h).
#include "scan_backward.h"

namespace merit {

template hipError_t scan_backward_of<float>(const ScanParams &p, hipStream_t s);

}  // namespace merit
