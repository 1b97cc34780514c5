// The bf16 d = 128 passes between sequences of two lengths, with the instruction scheduler
// of fb_passes_d128.hip.
#include "fb_ext_bob.h"

namespace fb {
FB_EXT_PASS1(bf16, 128)
FB_EXT_PASS2(bf16, 128)
}  // namespace fb
