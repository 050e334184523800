// The scan's backward pass on binary16 tensors (scan_backward.h).
#include "scan_backward.h"

namespace merit {

template hipError_t scan_backward_of<f16_t>(const ScanParams &p, hipStream_t s);

}  // namespace merit
