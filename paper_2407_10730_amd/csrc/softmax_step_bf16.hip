// softmax_step_bf16.hip -- softmax attention of few rows of a sequence, bf16 operands.
#include "softmax_device.h"

namespace cv {

hipError_t launch_softmax_step_bf16(const SoftArgs& a, bool vec, hipStream_t s) { return launch_softmax<uint16_t, true>(a, vec, s); }

}  // namespace cv
