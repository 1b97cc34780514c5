// Pass 1 between sequences of two lengths (bf16 d = 128 is in fb_ext_bob_d128.hip).
#include "fb_ext_bob.h"

namespace fb {
FB_EXT_PASS1(bf16, 32) FB_EXT_PASS1(bf16, 64) FB_EXT_PASS1(bf16, 256)
FB_EXT_PASS1(float, 32) FB_EXT_PASS1(float, 64) FB_EXT_PASS1(float, 128)
}  // namespace fb
