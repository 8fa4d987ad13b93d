// The experts' products for a token or a few: from fp16 activations in one kernel, bound by the stream of the active experts'
// weights and by what has to happen before its first request.
//
// Work is dealt as in the evenly split decode kernel (decode_split.h), but on the device, where the experts that have rows are
// known: their tiles (16 channels, all of K), times their row tiles of 16, make one list a part (8-bit and 4-bit channels; the
// blocks are shared out to the parts by bytes).
//  * Every block takes rounds of eight consecutive tiles, one a wave: the chip reads one window of the weights at a time.
//  * What is left after the last full round is dealt in quarter tiles (4 channels), evenly over the blocks, and inside a
//    block chunk by chunk over its waves.
//  * A chunk is four quantization groups of a tile, 4 KB of 4-bit or 8 KB of 8-bit weights.  The next chunk is in flight a wave
//    while one is consumed, issued and awaited by hand (async_loads.h); behind the end of the list come requests of one line,
//    so that every wait counts the same loads.
//  * Every block quantizes the activations for itself (the stand-alone quantizer's arithmetic, internal.h) while its first
//    weights are on their way, and keeps the codes in LDS.
//  * A chunk's contribution is added to the wave's LDS cell of the tile; after up to BATCH rounds and the rest the cells
//    (of a tile of the rest: all waves', in wave order) become results in one loop.
//  * The zero point is hoisted, sum a (q - z) = sum a q - z sum a, sum a from an MFMA against ones.  Scales per (token,
//    group): their products with the weights' from one fp16 MFMA a group, in the accumulators' layout.
// What comes before the first request (3.2 us by clock stamps, of the 11.4 of a token whose four experts have 26 MB) is as much of the
// time on small layers as the weights: every thread loads one expert's offsets and table entry at once, those with rows go into LDS one
// after another, and the lanes of a wave then work out where its next 64 chunks lie, a chunk a lane; a request only reads that out of
// its lane.  With the search for a chunk's expert in every request a token took 1.9 us more.  Two chunks in flight a wave: three and four
// 0.2 to 1.3 us more.  Against the quantizer and the tiled kernel: experts_stream_covers.
#include <algorithm>
#include <type_traits>

#include "async_loads.h"
#include "epilogue.h"
#include "experts.h"

namespace mixllm {

namespace {

constexpr int NW = 8, NT = NW * 64;
constexpr int BATCH = 4;         // rounds whose cells LDS holds at once
constexpr int MAX_REST = 9;      // virtual tiles of a block's last, partial round: less than eight tiles, cut at both ends
constexpr int RING = 2;          // chunks requested and not yet consumed
constexpr int MAX_PLACES = 128;  // rows, and so experts with rows, whose description lies in LDS
constexpr int MAX_VALUES = 16 * 1024;          // fp16 activations: four 16-byte loads a thread
constexpr int PIECES = MAX_VALUES / 8 / NT;
constexpr int A_PAD = 16;        // bytes added to every staged row of codes

template <int I, int N, typename F>
__device__ inline void sfor(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        sfor<I + 1, N>(f);
    }
}
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// one chunk in flight
template <bool PART8>
struct Slot {
    v4i w[4][PART8 ? 2 : 1];
    uint2 s;        // 4 fp16 scales of the lane's channel
    uint32_t z;     // 4 zero points (4-bit), or the fp16 channel scale (8-bit with one a channel)
};
template <int N, bool PART8>
__device__ inline void await_slot(Slot<PART8> &k)
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        asm volatile("" : "+v"(k.w[u][0]));
        if constexpr (PART8) asm volatile("" : "+v"(k.w[u][1]));
    }
    asm volatile("" : "+v"(k.s), "+v"(k.z));
}

// an expert with rows
struct Active {
    ExpertEntry x;
    int expert, first, count, unused;
};
static_assert(sizeof(ExpertEntry) == 64 && sizeof(Active) == 80, "entries are moved sixteen bytes at a time");
struct Shared {
    float red[BATCH + MAX_REST][NW][4][64];
    Active active[MAX_PLACES];
    int pre[2][MAX_PLACES];            // tiles of the active experts before, in the 4-bit and in the 8-bit part
    int tok[MAX_PLACES];               // places -> rows of the activations
    float sa[MAX_PLACES];              // ... and their scales (one per token)
    uint32_t rowmax[MAX_PLACES];       // scales per token: largest magnitudes of the rows as float bits
    unsigned long long sums[NW];
    unsigned long long limit;          // tiles of the first MAX_PLACES active experts, where lists name more
    int ranks[NW];
    uint16_t scales[MAX_VALUES / G];   // scales per group: [M][ng] fp16
    __attribute__((aligned(16))) int8_t codes[MAX_VALUES + MAX_PLACES * A_PAD];   // [M][K + A_PAD]
};

__device__ inline int at(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
template <typename T>
__device__ inline T *at(T *p, int l)
{
    const uint64_t b = (uint64_t)p;
    return spaced((T *)((uint64_t)(uint32_t)at((int)(uint32_t)b, l) | (uint64_t)(uint32_t)at((int)(uint32_t)(b >> 32), l) << 32));
}

// (a pointer out of LDS could be to anything, for the compiler: these are in global memory)
__device__ inline const __attribute__((address_space(1))) int32_t *channels(const int32_t *p) { return (const __attribute__((address_space(1))) int32_t *)p; }

struct Tile {   // a virtual tile
    const uint8_t *w;           // its packed tile
    const half_t *s;            // scales of its first row
    const uint8_t *z;           // zero points of its first row
    const int32_t *perm;        // channel of its first row
    int expert, first, count;   // the expert's places
    int row0;                   // first row of the row tile
    int rows;                   // channels of the tile that are there
    int quarters;               // qa + 8 qb: quarters [qa, qb) are this block's
};

template <bool ACT_PT, bool PART8, bool GROUPED8, typename STAGE>
__device__ inline void stream_block(const LinearParams &p, int b, int nblk, int U, int nactive, unsigned magic, Shared &m, STAGE &&stage)
{
    constexpr int GB = PART8 ? 2048 : 1024;   // bytes of one group of one tile
    constexpr int NL = (PART8 ? 8 : 4) + (PART8 ? 1 : 2);   // loads of a chunk
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), c = lane & 15, ks = lane >> 4;
    const int ng = p.ng, ngp = p.ngp, nquads = (ng + 3) / 4, xstride = p.K + A_PAD;

    const int rounds = uniform(U / (NW * nblk)), left0 = rounds * NW * nblk;   // U: tiles of this part
    // quarter tiles after the last full round, fewer than 32 nblk of them: block b begins behind b shares (exact products, a
    // rounding that is the same in every block, nothing lost at the end)
    const int left = 4 * (U - left0);
    const float share = (float)left * recip((float)nblk);
    auto begin = [&](int of) { return of == nblk ? left : min(left, (int)((float)of * share)); };
    const int lo = 4 * left0 + uniform(begin(b)), hi = 4 * left0 + uniform(begin(b + 1));
    const int nrest = hi > lo ? ((hi - 1) >> 2) - (lo >> 2) + 1 : 0;

    const int search = nactive > 1 ? 1 << (31 - __builtin_clz(nactive - 1)) : 0;
    auto over_quads = [&](int j) { return nquads == 1 ? j : (int)__umulhi((unsigned)j, magic); };   // j / nquads

    // virtual tile `i` of this wave, every lane its own: the tile of round i, or tile i - rounds of the rest
    auto describe = [&](int i) {
        Tile t;
        const bool rest = i >= rounds;
        const int unit = rest ? (lo >> 2) + (i - rounds) : (i * nblk + b) * NW + wave;
        t.quarters = rest ? (i == rounds ? lo & 3 : 0) + 8 * (unit == (hi - 1) >> 2 ? ((hi - 1) & 3) + 1 : 4) : 8 * 4;
        int e = 0;   // the last active expert whose tiles begin at or before the unit: among e .. e + 2 d - 1
#pragma unroll 1
        for (int d = search; d > 0; d /= 2)
            if (e + d < nactive && m.pre[PART8][e + d] <= unit) e += d;
        const Active &x = m.active[e];
        const int rt = (x.count + 15) / 16, local = max(unit - m.pre[PART8][e], 0);
        int tile = local;
        if (rt > 1) tile = local / rt;
        tile = max(min(tile, (PART8 ? x.x.ntiles8 : x.x.ntiles4) - 1), 0);   // (a tile that is there, whatever the lists say)
        t.expert = x.expert;
        t.first = x.first;
        t.count = x.count;
        t.row0 = 16 * min(local - tile * rt, rt - 1);
        t.w = (PART8 ? (const uint8_t *)x.x.w8 : x.x.w4) + (size_t)tile * ng * GB;
        t.s = (PART8 ? x.x.s8 : x.x.s4) + (size_t)tile * TILE_N * (PART8 && !GROUPED8 ? 1 : ngp);
        t.z = x.x.z4 + (size_t)tile * TILE_N * (ngp / 2);
        t.perm = x.x.perm + (PART8 ? 0 : x.x.n8) + tile * TILE_N;
        t.rows = min(TILE_N, (PART8 ? x.x.n8 : x.x.n4) - tile * TILE_N);
        return t;
    };

    // ---- a chunk's contribution to the sums of four rows (4 ks ..) of the lane's channel ----
    const v4i ones = {0x01010101, 0x01010101, 0x01010101, 0x01010101};
    auto compute = [&](int q, int row, const Slot<PART8> &k, float (&acc)[4]) {
        const float sh[4] = {half_bits_to_float(k.s.x & 0xffffu), half_bits_to_float(k.s.x >> 16), half_bits_to_float(k.s.y & 0xffffu),
                             half_bits_to_float(k.s.y >> 16)};
        const float sw_row = PART8 ? half_bits_to_float(k.z) : 0.0f;
        const int8_t *arow = m.codes + row * xstride + 16 * ks;
        uint32_t sa_bits = 0;   // fp16 activation scale of row lane & 15, group lane >> 4 of the chunk
        if constexpr (!ACT_PT) sa_bits = m.scales[row * ng + min(4 * q + ks, ng - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int8_t *ag = arow + min(4 * q + u, ng - 1) * G;
            const v4i a0 = *(const v4i *)ag, a1 = *(const v4i *)(ag + 64);
            v4i P;
            if constexpr (PART8) {
                P = __builtin_amdgcn_mfma_i32_16x16x64_i8(a0, k.w[u][0], v4i{0, 0, 0, 0}, 0, 0, 0);
                P = __builtin_amdgcn_mfma_i32_16x16x64_i8(a1, k.w[u][1], P, 0, 0, 0);
            } else {
                const v4i w = k.w[u][0];
                const int m4 = 0x0F0F0F0F;
                const v4i b0 = {w[0] & m4, (int)((uint32_t)w[0] >> 4) & m4, w[1] & m4, (int)((uint32_t)w[1] >> 4) & m4};
                const v4i b1 = {w[2] & m4, (int)((uint32_t)w[2] >> 4) & m4, w[3] & m4, (int)((uint32_t)w[3] >> 4) & m4};
                P = __builtin_amdgcn_mfma_i32_16x16x64_i8(a0, b0, v4i{0, 0, 0, 0}, 0, 0, 0);
                P = __builtin_amdgcn_mfma_i32_16x16x64_i8(a1, b1, P, 0, 0, 0);
                v4i S = __builtin_amdgcn_mfma_i32_16x16x64_i8(a0, ones, v4i{0, 0, 0, 0}, 0, 0, 0);
                S = __builtin_amdgcn_mfma_i32_16x16x64_i8(a1, ones, S, 0, 0, 0);
                const int z = (int)((k.z >> (4 * u)) & 15);
                // |z| <= 15 and |sum a| <= 128 * 127: the 24-bit multiply is exact
#pragma unroll
                for (int r = 0; r < 4; ++r) P[r] -= __mul24(z, S[r]);
            }
            const bool there = 4 * q + u < ng;   // (a group read again past the end of K contributes nothing)
            if constexpr (ACT_PT) {
                const float sw = !there ? 0.0f : (PART8 && !GROUPED8) ? sw_row : sh[u];
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf((float)P[r], sw, acc[r]);
            } else {
                // products of the two scales: row's in the lanes of group u, the channel's beside it, zeros elsewhere
                const uint32_t sw = !there || ks != u ? 0u : (PART8 && !GROUPED8) ? k.z & 0xffffu : ((u & 2) ? k.s.y : k.s.x) >> (16 * (u & 1)) & 0xffffu;
                const v4i A = {(int)(ks == u ? sa_bits : 0u), 0, 0, 0}, B = {(int)sw, 0, 0, 0};
                const v4f s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, A), __builtin_bit_cast(v8h, B), v4f{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf((float)P[r], s[r], acc[r]);
            }
        }
    };

    Slot<PART8> ring[RING];
    for (int r0 = 0;; r0 += BATCH) {
        // rounds r0 .. r0 + own - 1 and, with the last of them, the rest
        const int own = min(BATCH, rounds - r0);
        const bool with_rest = r0 + BATCH >= rounds;
        const int vts = own + (with_rest ? nrest : 0);
        const int n_own = own * nquads, n_rest = with_rest ? nrest * nquads : 0;   // (the rest's chunks are dealt to the waves one by one)
        const int n = n_own + (n_rest > wave ? (n_rest - wave + NW - 1) / NW : 0);
        for (int vt = 0; vt < vts; ++vt)   // this wave's cells start at zero
#pragma unroll
            for (int r = 0; r < 4; ++r) m.red[vt][wave][r][lane] = 0.0f;
        // the virtual tiles that this wave finishes, one a lane: its own, and every eighth of the rest; the first one's channels
        const int finishes = lane < own ? lane : own + wave + NW * (lane - own);
        Tile f;
        int ch0 = -1;
        for (int i0 = 0; i0 == 0 || i0 < n; i0 += 64) {
            const int cnt = min(64, n - i0);
            // this lane's chunk of the list: virtual tile of the batch and column
            const int mine = i0 + min(lane, max(cnt - 1, 0)), j = mine < n_own ? mine : wave + NW * (mine - n_own);
            const int jq = over_quads(j), vt_l = (mine < n_own ? 0 : own) + jq, q_l = j - jq * nquads;
            Tile t = describe(r0 + vt_l);
            t.w += (size_t)(4 * q_l) * GB;
            if constexpr (!PART8 || GROUPED8) t.s += 4 * q_l;
            t.z += 2 * q_l;
            const int last_l = ng - 1 - 4 * q_l;   // at the ragged end of K the last group is read again (its scale counts as zero)
            const int where_l = vt_l + 32 * q_l;
            auto request = [&](int i, Slot<PART8> &k) {   // (behind the end: the last chunk's first line)
                const int l = min(i, cnt - 1), last = at(last_l, l), quarters = at(t.quarters, l);
                // (quarters that another block takes are read as the nearest of this one's)
                const int c_row = 4 * min(max(c >> 2, quarters & 7), (quarters >> 3) - 1) + (c & 3);
                const uint32_t w_voff = i < cnt ? (uint32_t)(c_row + 16 * ks) * 16u : 0u;
                const uint8_t *wb = at(t.w, l);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint8_t *wu = wb + (size_t)min(u, last) * GB;
                    load_reg16_nt<0>(k.w[u][0], w_voff, wu);
                    if constexpr (PART8) load_reg16_nt<1024>(k.w[u][1], w_voff, wu);
                }
                k.s = make_uint2(0, 0);
                k.z = 0;
                if constexpr (!PART8) {
                    load_reg8(k.s, (uint32_t)(c_row * ngp * 2), at(t.s, l));
                    load_reg_u16(k.z, (uint32_t)(c_row * (ngp / 2)), at(t.z, l));
                } else if constexpr (GROUPED8)
                    load_reg8(k.s, (uint32_t)(c_row * ngp * 2), at(t.s, l));
                else
                    load_reg_u16(k.z, (uint32_t)(c_row * 2), at(t.s, l));
            };
            if (cnt > 0) sfor<0, RING - 1>([&](auto dc) { request(decltype(dc)::value, ring[decltype(dc)::value]); });
            if (i0 == 0) {   // (the weights are on their way)
                f = describe(r0 + min(finishes, max(vts - 1, 0)));
                if (vts > 0) ch0 = channels(at(f.perm, 0))[min(c, at(f.rows, 0) - 1)];
            }
            if (r0 == 0 && i0 == 0) {
                stage();
                lds_barrier();
            }
            for (int i = 0; i < cnt; i += RING)
                sfor<0, RING>([&](auto dc) {
                    constexpr int d = decltype(dc)::value;
                    request(i + d + RING - 1, ring[(d + RING - 1) % RING]);
                    await_slot<(RING - 1) * NL>(ring[d]);
                    if (i + d < cnt) {
                        const int l = i + d, where = at(where_l, l), vt = where & 31;
                        float part[4] = {};
                        const int row = m.tok[at(t.first, l) + min(at(t.row0, l) + c, at(t.count, l) - 1)];
                        compute(where >> 5, row, ring[d], part);
#pragma unroll
                        for (int r = 0; r < 4; ++r) m.red[vt][wave][r][lane] += part[r];
                    }
                });
            // nothing may still be on its way into a register when the registers get other uses
            sfor<0, RING>([&](auto dc) { await_slot<0>(ring[decltype(dc)::value]); });
        }
        if (n_rest > 0) lds_barrier();   // (the same for all waves)
        for (int i = 0;; ++i) {
            const int vt = i < own ? i : own + wave + NW * (i - own);
            if (vt >= vts) break;
            const int rows = at(f.rows, i), first = at(f.first, i), count = at(f.count, i), quarters = at(f.quarters, i), m0 = at(f.row0, i) + 4 * ks;
            const bool valid = c < rows && (c >> 2) >= (quarters & 7) && (c >> 2) < (quarters >> 3);
            const int ch = i == 0 ? ch0 : channels(at(f.perm, i))[min(c, rows - 1)];
            const int first_cell = vt < own ? wave : 0, cells = vt < own ? 1 : NW;
            float v[4] = {};
            for (int w = first_cell; w < first_cell + cells; ++w)
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] += m.red[vt][w][r][lane];
            if constexpr (ACT_PT) {
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] *= m.sa[first + min(m0 + r, count - 1)];
            }
            LinearParams q = p;
            q.M = count;
            q.y = p.y + (size_t)first * (p.ep.gated ? p.N / 2 : p.N);
            if (p.ep.bias) q.ep.bias = p.ep.bias + (size_t)at(f.expert, i) * p.N;
            store_rows(q, v, m0, valid ? ch : -1);
        }
        if (with_rest) break;   // (no barrier before the next batch: until the rest, a wave reads no cells but its own)
    }
}

template <bool ACT_PT, bool W8PC>
__global__ __launch_bounds__(NT) void experts_stream_kernel(LinearParams p, ExpertsArgs a, unsigned magic)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    Shared &m = *(Shared *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // what is needed from memory first is requested first: activations, rows and layers of the experts, places
    const int npiece = p.M * (p.K / 8), per_row = p.K / 8;
    h8 xv[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
        if (j * NT < npiece) xv[j] = ((const h8 *)p.x)[min(tid + NT * j, npiece - 1)];
    int tok = 0;
    if (tid < a.places) tok = token_row<true>(p, tid);
    int nactive = 0;
    unsigned long long before = 0;   // tiles of both parts, 32 bits each
    for (int e0 = 0; e0 < a.E; e0 += NT) {
        const int e = e0 + tid;
        const ExpertEntry *entry = a.table + min(e, a.E - 1);
        const uint4 words0 = ((const uint4 *)entry)[0], words1 = ((const uint4 *)entry)[1], words2 = ((const uint4 *)entry)[2], words3 = ((const uint4 *)entry)[3];
        int first, count;
        expert_rows(a, min(e, a.E - 1), first, count);
        if (e >= a.E) count = 0;
        const int rt = (count + 15) / 16;
        // (the last sixteen bytes of an entry: n8, n4, ntiles8, ntiles4)
        const unsigned long long tiles = (unsigned long long)(rt * words3.w) | (unsigned long long)(rt * words3.z) << 32;
        const unsigned long long here = __ballot(count > 0);
        unsigned long long x = tiles;
        if (here) {
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const unsigned long long o = __shfl_up(x, d);
                if (lane >= d) x += o;
            }
        }
        if (lane == 63) {
            m.sums[wave] = x;
            m.ranks[wave] = __popcll(here);
        }
        __syncthreads();
        int rank = nactive + __popcll(here & ((1ull << lane) - 1)), all_ranks = 0;
        unsigned long long all = 0;
        x += before - tiles;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < wave) {
                x += m.sums[w];
                rank += m.ranks[w];
            }
            all += m.sums[w];
            all_ranks += m.ranks[w];
        }
        if (count > 0 && rank == MAX_PLACES) m.limit = x;   // (as long as the offsets ascend there are no more such experts than places)
        if (count > 0 && rank < MAX_PLACES) {
            uint4 *cell = (uint4 *)&m.active[rank].x;
            cell[0] = words0;
            cell[1] = words1;
            cell[2] = words2;
            cell[3] = words3;
            m.active[rank].expert = e;
            m.active[rank].first = first;
            m.active[rank].count = count;
            m.pre[0][rank] = (int)(uint32_t)x;
            m.pre[1][rank] = (int)(uint32_t)(x >> 32);
        }
        before += all;
        nactive += all_ranks;
        if (e0 + NT < a.E) __syncthreads();
    }
    nactive = uniform(nactive);
    if (tid < a.places) {
        m.tok[tid] = tok;
        m.rowmax[tid] = 0;   // (as many rows as places at most)
    }
    __syncthreads();
    if (nactive > MAX_PLACES) {
        nactive = MAX_PLACES;
        before = m.limit;
    }
    const unsigned most = (unsigned)a.places * ((unsigned)(p.N + 30) / 16 + 1);
    const int U4 = uniform((int)min((uint32_t)before, most)), U8 = uniform((int)min((uint32_t)(before >> 32), most)), B = gridDim.x;
    auto stage = [&]() {
        // largest magnitudes: the 16 lanes that hold a quantization group find it among themselves (K is a multiple of 128, so such
        // a run of 16 pieces lies in one row and one group, and is loaded completely or not at all)
        float group_max[PIECES];
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
            if (j * NT < npiece) {
                asm volatile("" : "+v"(xv[j]));   // (none of this is worked out before the first request)
                u16x2 am = {0, 0};
                absmax8(xv[j], am);
                group_max[j] = row16_max(absmax_of(am));
                const int i = tid + NT * j;
                if (ACT_PT && i < npiece && (lane & 15) == 0) atomicMax(&m.rowmax[i / per_row], __builtin_bit_cast(uint32_t, group_max[j]));
            }
        if constexpr (ACT_PT) lds_barrier();
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int i = tid + NT * j;
            if (j * NT < npiece && i < npiece) {
                const int row = i / per_row, pos = i - row * per_row;
                const half_t s16 = store_scale((ACT_PT ? __builtin_bit_cast(float, m.rowmax[row]) : group_max[j]) / 127.0f);
                const float s = (float)s16;
                *(uint2 *)(m.codes + row * (p.K + A_PAD) + pos * 8) = quant8(xv[j], s, recip(s));
                if (!ACT_PT && (lane & 15) == 0) m.scales[row * p.ng + (pos >> 4)] = __builtin_bit_cast(uint16_t, s16);
            }
        }
        if constexpr (ACT_PT)
            if (tid < a.places) m.sa[tid] = (float)store_scale(__builtin_bit_cast(float, m.rowmax[m.tok[tid]]) / 127.0f);
    };
    // blocks of the 8-bit part, whose tiles have twice the bytes (every block comes to the same number, whatever its rounding)
    int nb8 = U8 == 0 ? 0 : (int)(2.0f * (float)U8 * (float)B * recip(2.0f * (float)U8 + (float)U4) + 0.5f);
    if (U8 > 0) nb8 = min(max(nb8, 1), B);
    if (U4 > 0) nb8 = min(nb8, B - 1);
    nb8 = uniform(nb8);
    if ((int)blockIdx.x < nb8) stream_block<ACT_PT, true, !W8PC>(p, blockIdx.x, nb8, U8, nactive, magic, m, stage);
    else if (U4 > 0) stream_block<ACT_PT, false, false>(p, blockIdx.x - nb8, B - nb8, U4, nactive, magic, m, stage);
}

}  // namespace

// Where this kernel takes the call: while the activations fit the registers they are quantized from (M K <= MAX_VALUES), but for more than
// eight rows of K <= 2048 with one scale a row, where the quantizer's launch and the tiled kernel are ahead.  us, this kernel and those two,
// 64 experts, other ones from call to call, N = 4096 (1024):
//   4 rows                                        8 rows                              32 rows
//   K =  512    8.6 and  8.7  (8.0 and  7.8)       9.5 and  9.5  (8.2 and  8.6)       14.9 and 14.6  ( 9.9 and  9.0)
//   K = 1408    9.8 and 10.9  (8.5 and 10.6)      12.7 and 12.1  (9.0 and 10.9)       23.8 and 22.5  (12.4 and 11.5)
//   K = 2048   11.0 and 12.6  (8.8 and 11.8)      15.0 and 15.4  (9.2 and 12.0)       30.0 and 29.4  (14.0 and 13.0)
//   K = 4096   14.4 and 18.8  (9.2 and 16.3)      21.1 and 24.4 (11.6 and 16.6)       50.6 and 53.8  (20.1 and 18.6)
// K = 14336, one token of four experts 32.9 and 52.3; 64 rows of K = 1024 28.5 and 24.2, 128 rows 34.3 and 30.0.  With scales per 128
// channels it is level or ahead at most sizes (K = 1408, 4, 8, 32 rows: 9.9 and 11.8, 12.8 and 13.2, 23.7 and 24.9; 16 to 64 rows of K <= 512 and N = 1024
// 4 to 10 % behind).  A token's four experts of K = 4096, N = 2816 12.4 and 18.4, two tokens' 16.8 and 19.0, four tokens' 24.9 and 26.2.
bool experts_stream_covers(const LinearParams &p, const ExpertsArgs &a)
{
    // tiles of a part, in quarters, in 32 bits: every place may be a row tile of its own, and every expert may have all places in
    // lists that overlap
    const long tiles = std::max((long)a.places, (long)a.E * ((a.places + 15) / 16)) * ((p.N + 30) / 16 + 1);
    if (a.places > MAX_PLACES || p.M > MAX_PLACES || (size_t)p.M * p.K > (size_t)MAX_VALUES || 4 * tiles >= (1l << 31)) return false;
    return !(p.act_per_token && a.places > 8 && p.K <= 2048);
}

int launch_experts_stream(const LinearParams &p, const ExpertsArgs &a, hipStream_t st)
{
    auto go = [&](auto kernel) {
        if (int e = ensure_dynamic_lds((const void *)kernel, sizeof(Shared))) return e;
        const int nquads = (p.ng + 3) / 4;
        hipLaunchKernelGGL(kernel, dim3(cu_count()), dim3(NT), sizeof(Shared), st, p, a, (unsigned)(((1ull << 32) + nquads - 1) / nquads));
        return (int)hipGetLastError();
    };
    if (p.act_per_token) return p.w8_per_channel ? go(experts_stream_kernel<true, true>) : go(experts_stream_kernel<true, false>);
    return p.w8_per_channel ? go(experts_stream_kernel<false, true>) : go(experts_stream_kernel<false, false>);
}

}  // namespace mixllm
