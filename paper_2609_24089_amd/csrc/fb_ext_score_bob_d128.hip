// The bf16 d = 128 passes over capped scores, distance biases and spans, with the instruction
// scheduler of fb_passes_d128.hip.
#include "fb_ext_score_bob.h"

namespace fb {
FB_SCORE_PASS1(bf16, 128)
FB_SCORE_PASS2(bf16, 128)
}  // namespace fb
