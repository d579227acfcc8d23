// softmax_prompt_f32.hip -- softmax attention of many rows of a sequence, fp32 operands on the fp32 matrix instruction.
#include "softmax_device.h"

namespace cv {

hipError_t launch_softmax_prompt_f32(const SoftArgs& a, bool vec, hipStream_t s) { return launch_softmax<float, false>(a, vec, s); }

}  // namespace cv
