// softmax_bf16.hip -- softmax attention, bf16 operands.
#include "softmax_device.h"

namespace cv {

hipError_t launch_softmax_bf16(const SoftArgs& a, bool vec, hipStream_t s) { return launch_softmax<uint16_t, 64>(a, vec, s); }

}  // namespace cv
