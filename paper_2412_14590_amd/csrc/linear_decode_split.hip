// The evenly split decode kernel (decode_split.h) as the plain linear, which shapes it takes, and its plan.
#include "decode_split.h"

namespace mixllm {

bool decode_split_covers(const LinearParams &p)
{
    Plan pl;
    return make_plan(p, pl);
}

// the launch plan as six integers (blocks of the 8-bit part, of the 4-bit part, virtual tiles an
// LDS cell area covers, bytes of LDS, windows the activations are staged in, chunk columns - 512
// values of K - per window), for the host-side test of the work split
bool decode_split_plan(const LinearParams &p, int out[6])
{
    Plan pl;
    if (!make_plan(p, pl)) return false;
    out[0] = pl.nblk8;
    out[1] = pl.nblk4;
    out[2] = pl.tcap;
    out[3] = (int)pl.lds_bytes;
    out[4] = pl.nwin;
    out[5] = pl.wq;
    return true;
}

int launch_linear_decode_split(const LinearParams &p, hipStream_t st) { return launch_split<false>(p, st); }

}  // namespace mixllm
