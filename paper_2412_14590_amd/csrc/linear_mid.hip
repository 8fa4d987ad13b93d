// The kernel for a few dozen tokens (mid.h) as the plain linear, which shapes it takes, and its plan.
#include "mid.h"

namespace mixllm {

bool mid_covers(const LinearParams &p)
{
    if (p.M < 1 || p.M > 64 || p.ng < 1 || p.x) return false;
    // one activation scale per (token, group): up to 32 tokens (with four token tiles per wave the extra
    // scale reads do not fit the register file next to the weight ring: the tiled kernel takes those)
    if (!p.act_per_token && !p.P && p.M > 32) return false;
    if (lds_bytes_of(p) > LDS_LIMIT) return false;
    // 32-bit lane offsets inside the activation, weight and metadata arrays
    const size_t two_tiles = 2 * (size_t)p.ng * 2048 + 2048;
    if ((size_t)p.M * p.K >= (1ull << 31) || two_tiles >= (1ull << 31)) return false;
    if (4ll * std::max(p.ntiles8, p.ntiles4) * 4096 >= (1ll << 31)) return false;
    return p.ntiles8 + p.ntiles4 > 0;
}

// the launch plan as five integers (blocks of the 8-bit part, of the 4-bit part, quarter tiles per
// virtual tile of either part, bytes of LDS), for the host-side test of the work split
bool mid_plan(const LinearParams &p, int out[5])
{
    if (!mid_covers(p)) return false;
    MidArgs a;
    size_t lds_bytes;
    mid_args(p, a, lds_bytes);
    out[0] = a.nblk8;
    out[1] = a.nblk4;
    out[2] = a.qv8;
    out[3] = a.qv4;
    out[4] = (int)lds_bytes;
    return true;
}

int launch_linear_mid(const LinearParams &p, hipStream_t st) { return launch_mid<false>(p, st); }

}  // namespace mixllm
