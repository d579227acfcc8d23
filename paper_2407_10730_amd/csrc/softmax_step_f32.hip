// softmax_step_f32.hip -- softmax attention of few rows of a sequence, fp32 operands on the fp32 matrix instruction.
#include "softmax_device.h"

namespace cv {

hipError_t launch_softmax_step_f32(const SoftArgs& a, bool vec, hipStream_t s) { return launch_softmax<float, true>(a, vec, s); }

}  // namespace cv
