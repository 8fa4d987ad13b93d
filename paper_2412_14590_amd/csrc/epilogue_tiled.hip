// The tiled kernel and the tiles cut along K (tiled.h) with an epilogue (epilogue.h).
#include "tiled.h"

namespace mixllm {

int launch_tiled_epilogue(const LinearParams &p, hipStream_t st) { return launch_tiled<true>(p, st); }

int launch_slices_epilogue(const LinearParams &p, hipStream_t st) { return launch_slices<true>(p, st); }

}  // namespace mixllm
