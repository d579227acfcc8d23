// softmax_prompt_bf16.hip -- softmax attention of many rows of a sequence, bf16 operands.
#include "softmax_device.h"

namespace cv {

hipError_t launch_softmax_prompt_bf16(const SoftArgs& a, bool vec, hipStream_t s) { return launch_softmax<uint16_t, false>(a, vec, s); }

}  // namespace cv
