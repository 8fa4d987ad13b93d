// The tiled kernel and the tiles cut along K (tiled.h) as the plain linear, which shapes they take, and their plans.
#include "tiled.h"

namespace mixllm {

#ifdef MIXLLM_STAMPS
extern "C" int mixllm_debug_set_stamps(void *stamps)
{
    return (int)hipMemcpyToSymbol(HIP_SYMBOL(g_stamps), &stamps, sizeof stamps);
}
#endif

// Shapes the kernel takes: lanes address activations, packed weights and metadata with 32-bit byte
// offsets; a caller-chosen block shape must exist for the scale granularity.
bool prefill_covers(const LinearParams &p)
{
    const size_t lim = (size_t)1 << 31;
    if ((size_t)p.M * (size_t)p.K >= lim || (size_t)p.ntiles4 * TILE_N * (size_t)p.K / 2 >= lim ||
        (size_t)p.ntiles8 * TILE_N * (size_t)p.K >= lim)
        return false;
    return p.M >= 1 && p.N >= 1 && token_tiles_per_wave(p, 0) != 0;
}

// true when the kernel, given `p.partials_cap` bytes of scratch, would split K
bool prefill_would_split(const LinearParams &p)
{
    int qpp;
    return prefill_covers(p) && p.partials && choose_kparts(p, token_tiles_per_wave(p, p.partials_cap), p.partials_cap, qpp) > 1;
}

size_t prefill_scratch_bytes(const LinearParams &p)
{
    if (!prefill_covers(p)) return 0;
    int qpp;
    const int kp = choose_kparts(p, token_tiles_per_wave(p, ~(size_t)0), ~(size_t)0, qpp);
    return kp > 1 ? (size_t)kp * p.M * p.np * sizeof(float) : 0;
}

int launch_linear_prefill(const LinearParams &p, hipStream_t st) { return launch_tiled<false>(p, st); }

int launch_linear_slices(const LinearParams &p, hipStream_t st) { return launch_slices<false>(p, st); }

// Where linear_slices_kernel takes over: from 17 tokens (up to 16 the decode kernels are ahead, K = N = 4096: 7.2 us
// against 7.8), with a group of 4 quantization groups or more for each of its waves, while all its blocks run at once.
// The lines lie where the two sides change places, measured in turn on one machine with every launch's weights from HBM
// and 10 % 8-bit channels: 5900 pairs, 17 to 400 tokens, K = 1664 .. 28672, both granularities of the activation scales
// ("grouped" = one per token and group).  A factor is the time of the kernel that otherwise takes the call over the slices'.
//  * One block a CU.  What counts is the busiest XCD: 256 tiles make 264 blocks in eight equal ranges of either part, and the
//    second block on some CUs costs 30 % (K = 4096 at 17 tokens: 8.1 us with 248 blocks, 10.9 with 264).  Factor 1.2 to 3.7
//    at any K where the other side does not split K over blocks (up to 32 tokens it does beyond K = 8192).  Against a split,
//    K = 8192 0.93 to 1.7, grouped 0.83 to 1.33; otherwise from 7/16 of the CUs on: grouped 0.91 to 1.4, else 0.95 to 1.5, below
//    that 0.64 to 1.2 (K = 14336 at 17 / 32 tokens: 120 blocks 1.12 / 1.01, 104 blocks 0.90 / 0.78).  Never at K = 28672
//    (0.43 to 1.27).  (Two places where the split is ahead stay with the slices, because calls there give the same bits with
//    scratch and without: grouped, K = 8192, fewer than 96 blocks, 33 to 64 tokens, and, beyond K = 8192, up to 24
//    tokens and three blocks an XCD, 0.68 to 1.05.)
//  * Two blocks a CU, one token tile: the path for a few dozen tokens reads the weights evenly and is level or ahead
//    (K = 8192, 264 to 392 blocks: 0.97 to 1.00 at 17 tokens, 0.89 to 0.95 at 32) until its blocks hold more virtual tiles than
//    a CU has SIMDs: more weights than four 4-bit tiles a CU (K = 8192, 472 blocks 1.08 / 1.02, 480 blocks 1.37 / 1.26; K = 2048
//    1.15 / 1.12).  Grouped, up to 24 tokens and K = 8192, 0.98 to 1.14 before that as well (at 32 tokens 0.92 to 1.04).
//  * Two blocks a CU, more tokens: 1.02 to 2.4.  Against a split 0.96 to 1.4 at K = 8192, grouped from 3/2 blocks a CU on
//    (1.01 to 1.29, 296 blocks 0.87 to 0.95); beyond that K 0.60 to 1.2.
//  * A few blocks more than two a CU, which run by themselves at the end: from K = 4096 on, one more an XCD (0.99 to 1.19), two
//    from 65 tokens on or grouped (1.03 to 1.42; else 0.85 to 1.15).  Shorter K 0.85 to 1.0; one token tile 0.79 to 1.16.
// Beyond 64 tokens a call that brings the scratch to split K over blocks gets that split although the slices are ahead at
// K = 8192 (0.87 to 1.7): its results are those of the tiled path by name, bit for bit, which is kept.
bool slices_pay(const LinearParams &p)
{
    if (p.P || p.S || p.M <= 16 || p.ng < 4 * SLICES - 3 || !prefill_covers(p)) return false;
    const bool split = prefill_would_split(p), grouped = !p.act_per_token;
    if (p.M > 64 && split) return false;
    const long blocks = slices_grid(p).blocks(), cus = cu_count();
    if (blocks <= cus) {
        if (!split || p.ng <= 64) return true;
        return p.ng <= 112 && (16 * blocks > 7 * cus || (p.M <= 24 && blocks <= 24));
    }
    if (split && (p.ng > 64 || (grouped && p.M > 32 && 2 * blocks < 3 * cus))) return false;
    if (p.M <= 32) {
        const bool many_tiles = p.ntiles4 > 0 && p.ntiles4 + 2L * p.ntiles8 > 4 * cus;
        return blocks <= 2 * cus && (many_tiles || (grouped && p.M <= 24 && p.ng <= 64));
    }
    return blocks <= 2 * cus + (p.ng < 32 ? 0 : p.M <= 64 && !grouped ? 8 : 16);
}

// the launch plan as six integers (token tiles, channel tiles of either part, blocks, slices, bytes of LDS)
void slices_plan(const LinearParams &p, int out[6])
{
    const SlicesGrid g = slices_grid(p);
    out[0] = g.nbm;
    out[1] = g.nb8;
    out[2] = g.nb4;
    out[3] = g.blocks();
    out[4] = SLICES;
    out[5] = (int)slices_lds_bytes(p.act_per_token);
}

// the launch plan as thirteen integers (token rows and channels of a block tile of the 4-bit part, its
// token tiles, channel tiles of the 8-bit and of the 4-bit part, blocks launched per K part, token tiles
// per band of the 4-bit part, bytes of LDS, K parts, groups per K part, then token rows, token tiles and
// token tiles per band of the 8-bit part), for the host-side test of the block -> tile mapping
bool prefill_plan(const LinearParams &p, int out[13])
{
    if (!prefill_covers(p)) return false;
    const int tm = token_tiles_per_wave(p, ~(size_t)0);   // (the plan of a launch that has the scratch to split K)
    const int BM = 32 * tm, BN = tm == 4 ? 32 * MIXLLM_PREFILL_WN_LARGE : 128;
    const PrefillGrid g = grid_of(p, BM, BN);
    out[0] = BM;
    out[1] = BN;
    out[2] = g.nbm4;
    out[3] = g.nb8;
    out[4] = g.nb4;
    out[5] = (g.per4 + g.per8) * 8;
    out[6] = g.band4;
    out[7] = NSTAGE * BM * G + (int)token_scale_bytes(!p.act_per_token && !p.P, BM);   // (p.P is never set here)
    int qpp;
    out[8] = choose_kparts(p, tm, ~(size_t)0, qpp);   // blocks sharing a K range when the caller brings the scratch for it
    out[9] = 4 * qpp;                                 // quantization groups per part
    out[10] = g.bm8;                                  // token rows, token tiles and token tiles per band of the 8-bit part
    out[11] = g.nbm8;
    out[12] = g.band8;
    return true;
}

}  // namespace mixllm
