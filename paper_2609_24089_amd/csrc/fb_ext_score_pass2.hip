// Pass 2 over capped scores, distance biases and spans (bf16 d = 128 is in
// fb_ext_score_bob_d128.hip).
#include "fb_ext_score_bob.h"

namespace fb {
FB_SCORE_PASS2(bf16, 32) FB_SCORE_PASS2(bf16, 64) FB_SCORE_PASS2(bf16, 256)
FB_SCORE_PASS2(float, 32) FB_SCORE_PASS2(float, 64) FB_SCORE_PASS2(float, 128)
}  // namespace fb
