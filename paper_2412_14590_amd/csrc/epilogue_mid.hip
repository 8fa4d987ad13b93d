// The kernel for a few dozen tokens (mid.h) with an epilogue (epilogue.h).
#include "mid.h"

namespace mixllm {

int launch_mid_epilogue(const LinearParams &p, hipStream_t st) { return launch_mid<true>(p, st); }

}  // namespace mixllm
