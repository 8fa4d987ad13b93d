// The evenly split decode kernel (decode_split.h) with an epilogue (epilogue.h).
#include "decode_split.h"

namespace mixllm {

int launch_split_epilogue(const LinearParams &p, hipStream_t st) { return launch_split<true>(p, st); }

}  // namespace mixllm
