// The products of a layer of experts over the rows routed to them, and the weighted sum of every token's rows.
//
// The products run the tiles of the linear (tiled.h) - the same loads, matrix instructions, rescale and epilogue -
// on one expert's packed layer and rows a block.  Rows come through the route's list (the activations of a token are
// quantized and kept once, whatever the number of experts that read them) or lie one after another.  How many rows an
// expert has is known on the device only: the grid covers the most tiles that the rows could make, and every
// block finds its tile from the offsets by a sum over the experts.
#include <algorithm>

#include "experts.h"
#include "tiled.h"

namespace mixllm {

namespace {

constexpr long MAX_WORK_ITEMS = (1l << 32) - 1;   // blocks times threads of a launch, in x

constexpr int TABLE_CHUNK = 32;   // entries that travel as arguments of one launch
struct TableChunk {
    ExpertEntry entry[TABLE_CHUNK];
};
__global__ void experts_table_kernel(ExpertEntry *table, TableChunk chunk, int first, int n)
{
    if ((int)threadIdx.x < n) table[first + threadIdx.x] = chunk.entry[threadIdx.x];
}

// The tile of this block, and p made that of its expert.  The tiles of the 4-bit parts make one list, those of the 8-bit
// parts another: expert by expert, column by column, the row tiles of a column next to each other.  Blocks are dealt to the
// eight XCDs round robin; an XCD runs a contiguous eighth of either list, so that the blocks that share an expert's
// weights and rows share an L2, and ends on the cheaper 8-bit tiles.  (Columns dealt to the XCDs in turn share out the low
// last row tiles better, but every L2 then reads all rows: 4096 tokens, the products alone, 312 -> 333 us.)
struct TileOf {
    bool none, part8;
    int row0, bn;   // first row of the expert's, column of channels
    int left;       // rows from row0 on
};
template <int BM4, int BM8, int T16, bool ACT_PT>
static __device__ __forceinline__ TileOf find_tile(LinearParams &p, const ExpertsArgs &a)
{
    const int lane = threadIdx.x & 63;
    // tiles of expert e in either part
    auto tiles_of = [&](int e, int &t4, int &t8) {
        t4 = t8 = 0;
        if (e < a.E) {
            int first, count;
            expert_rows(a, e, first, count);
            t4 = (count + BM4 - 1) / BM4 * ((a.table[e].ntiles4 + T16 - 1) / T16);
            t8 = (count + BM8 - 1) / BM8 * ((a.table[e].ntiles8 + T16 - 1) / T16);
        }
    };
    int first4, first8;   // of the first 64 experts: kept, the others are read a second time below
    tiles_of(lane, first4, first8);
    int total4 = first4, total8 = first8;
    for (int e0 = 64; e0 < a.E; e0 += 64) {
        int t4, t8;
        tiles_of(e0 + lane, t4, t8);
        total4 += t4;
        total8 += t8;
    }
    total4 = uniform(__shfl(wave_scan(total4), 63));
    total8 = uniform(__shfl(wave_scan(total8), 63));
    const int per4 = (total4 + 7) / 8, per8 = (total8 + 7) / 8;
    const int xcd = blockIdx.x & 7, i = blockIdx.x >> 3;
    TileOf t;
    t.part8 = i >= per4;
    const int L = t.part8 ? xcd * per8 + (i - per4) : xcd * per4 + i;
    t.none = t.part8 ? (i - per4 >= per8 || L >= total8) : L >= total4;
    if (t.none) return t;
    int e = -1, before = 0;
    for (int e0 = 0, sum = 0; e0 < a.E; e0 += 64) {
        int t4 = first4, t8 = first8;
        if (e0 > 0) tiles_of(e0 + lane, t4, t8);
        const int own = t.part8 ? t8 : t4, upto = sum + wave_scan(own);
        const unsigned long long here = __ballot(own > 0 && L >= upto - own && L < upto);
        if (here) {
            const int l = __ffsll(here) - 1;
            e = uniform(e0 + l);
            before = uniform(__shfl(upto - own, l));
            break;
        }
        sum = uniform(__shfl(upto, 63));
    }
    t.none = e < 0;   // (lists that say so much that the sums overflow)
    if (t.none) return t;
    const ExpertEntry x = expert_entry(a, e);
    int first, count;
    expert_rows_uniform(a, e, first, count);
    p.w4 = x.w4;
    p.w8 = x.w8;
    p.s4 = x.s4;
    p.s8 = x.s8;
    p.z4 = x.z4;
    p.perm = x.perm;
    p.n8 = x.n8;
    p.n4 = x.n4;
    p.ntiles8 = x.ntiles8;
    p.ntiles4 = x.ntiles4;
    p.M = count;
    if (p.rows) p.rows += first;
    else {
        p.xq += (size_t)first * p.K;
        p.xscale += (size_t)first * (ACT_PT ? 1 : p.ng);
    }
    p.y += (size_t)first * (p.ep.gated ? p.N / 2 : p.N);
    if (p.ep.bias) p.ep.bias += (size_t)e * p.N;
    const int BM = t.part8 ? BM8 : BM4, nbm = (count + BM - 1) / BM, r = L - before;
    t.bn = uniform(r / nbm);
    t.row0 = (r - t.bn * nbm) * BM;
    t.left = count - t.row0;
    return t;
}

// Experts' rows come in any number: the last row tile of an expert is as low as its rows allow (half or a quarter of the others;
// the quarter is 32 rows).  4096 tokens to 4 of 64 experts each, K 4096, N 2816: 343 -> 325 us.
template <typename C, bool ACT_PT, bool W8PC>
__global__ __launch_bounds__(C::THREADS, 2) void experts_tiled_kernel(LinearParams p, ExpertsArgs a)
{
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    using C8 = typename C::Half;
    constexpr int T16 = C::BN / TILE_N;
    const TileOf t = find_tile<C::BM, C8::BM, T16, ACT_PT>(p, a);
    if (t.none) return;
    uint8_t *lds_a = smem;
    float *lds_sa = (float *)(smem + NSTAGE * C::A_STAGE);
    auto tile8 = [&](auto shape) {
        using S = decltype(shape);
        if constexpr (W8PC && ACT_PT)
            prefill_block_w8_channel_scale<S, ACT_PT, 0, true, true>(p, t.row0, t.bn * T16, 0, p.ng, 0, lds_a, lds_sa, smem);
        else
            prefill_block<S, 0, ACT_PT, true, !W8PC, true, true, true>(p, t.row0, t.bn * T16, 0, p.ng, 0, lds_a, lds_sa, smem);
    };
    auto tile4 = [&](auto shape) {
        using S = decltype(shape);
        prefill_block<S, 0, ACT_PT, false, false, true, true, true>(p, t.row0, t.bn * T16, 0, p.ng, 0, lds_a, lds_sa, smem);
    };
    auto pick = [&](auto top, auto &&tile) {
        constexpr int TM = decltype(top)::TM;
        if constexpr (TM > 1)
            if (t.left <= 32) return tile(Shape<C::WM, C::WN, 1, C::WD>{});
        if constexpr (TM > 2)
            if (t.left <= 64) return tile(Shape<C::WM, C::WN, 2, C::WD>{});
        tile(top);
    };
    if (t.part8) pick(C8{}, tile8);
    else pick(C{}, tile4);
}

// the most tiles, as blocks: every expert with rows may have a row tile that is not full; the 4-bit part is at most the layer, the
// 8-bit part the largest of any expert (a.n8).  Blocks without a tile live for a microsecond.
template <typename C>
long blocks_of(const LinearParams &p, const ExpertsArgs &a)
{
    const long busy = std::min(a.E, a.places);
    const long tiles4 = (a.places / C::BM + busy) * ((round_up(p.N, TILE_N) + C::BN - 1) / C::BN);
    const long tiles8 = (a.places / C::Half::BM + busy) * ((round_up(a.n8, TILE_N) + C::BN - 1) / C::BN);
    return 8 * ((tiles4 + 7) / 8 + (tiles8 + 7) / 8);
}

template <typename C>
int launch_experts_shape(const LinearParams &p, const ExpertsArgs &a, hipStream_t st)
{
    const long blocks = blocks_of<C>(p, a);
    auto go = [&](auto kernel, bool grouped) {
        const size_t lds = (size_t)NSTAGE * C::A_STAGE + token_scale_bytes(grouped, C::BM);
        if (int e = ensure_dynamic_lds((const void *)kernel, lds)) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(C::THREADS), lds, st, p, a);
        return (int)hipGetLastError();
    };
    if (p.act_per_token) return p.w8_per_channel ? go(experts_tiled_kernel<C, true, true>, false) : go(experts_tiled_kernel<C, true, false>, false);
    if constexpr (C::TM <= 2) return p.w8_per_channel ? go(experts_tiled_kernel<C, false, true>, true) : go(experts_tiled_kernel<C, false, false>, true);
    return (int)hipErrorInvalidValue;
}

// One token's columns a thread: 8 where rows and columns allow 16-byte accesses, else one.  Bound by memory: 4096 tokens of 4 rows of 4096
// columns and a residual, 201 MB, 30 us (6.7 TB/s, part of the rows still in the caches from the products).
template <int V>
__global__ __launch_bounds__(256) void experts_combine_kernel(int T, int k, int N, int places, const half_t *y, const float *weights,
                                                              const int32_t *slots, const half_t *residual, half_t *out)
{
    typedef half_t vec __attribute__((ext_vector_type(V)));
    const int n = (blockIdx.y * 256 + threadIdx.x) * V, t = blockIdx.x;   // (a grid may have 2^16 blocks in y only)
    if (n >= N) return;
    float sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) sum[v] = 0.0f;
    const size_t cell = (size_t)t * N + n;
    vec res = {};
    if (residual) res = *(const vec *)(residual + cell);
    for (int j = 0; j < k; ++j) {
        const int slot = slots[(size_t)t * k + j];
        const float w = weights[(size_t)t * k + j];
        if (slot < 0 || slot >= places) continue;
        const vec row = *(const vec *)(y + (size_t)slot * N + n);
#pragma unroll
        for (int v = 0; v < V; ++v) sum[v] = __builtin_fmaf(w, (float)row[v], sum[v]);
    }
    vec o;
#pragma unroll
    for (int v = 0; v < V; ++v) o[v] = (half_t)(sum[v] + (float)res[v]);
    *(vec *)(out + cell) = o;
}

}  // namespace

int launch_experts_table(int E, int N, const mixllm_expert *experts, ExpertEntry *table, hipStream_t st)
{
    for (int e0 = 0; e0 < E; e0 += TABLE_CHUNK) {
        TableChunk c{};
        const int n = std::min(TABLE_CHUNK, E - e0);
        for (int i = 0; i < n; ++i) {
            const mixllm_expert &x = experts[e0 + i];
            const int n4 = N - x.n8;
            c.entry[i] = ExpertEntry{(const uint8_t *)x.packed_w4, (const int8_t *)x.packed_w8, (const half_t *)x.scales4, (const half_t *)x.scales8,
                                     (const uint8_t *)x.zeros4, x.feature_perm, x.n8, n4, round_up(x.n8, TILE_N) / TILE_N, round_up(n4, TILE_N) / TILE_N};
        }
        hipLaunchKernelGGL(experts_table_kernel, dim3(1), dim3(64), 0, st, table, c, e0, n);
        if (hipError_t err = hipGetLastError()) return (int)err;
    }
    return (int)hipSuccess;
}

// lanes address activations and one expert's weights and metadata with 32-bit byte offsets, whatever its share of 8-bit channels
bool experts_cover(const LinearParams &p)
{
    const size_t lim = (size_t)1 << 31;
    return (size_t)p.M * p.K < lim && (size_t)(p.N + 30) * p.K < lim;
}

// The height of the row tiles, by the rows of an expert on average (which experts they go to is known on the device only).
// A higher tile reads the weights and unpacks them less often, a lower one starts sooner and shares out better.  64 experts,
// K 4096, N 2816, the products alone, us with 32, 64, 128 rows: mean 8: 76.5, 78.3, 83.7; 16: 85.8, 85.5, 94.1; 32: 101, 99, 107;
// 64: 145, 128, 130; 96: 189, 161, 158; 256: 414, 345, 317.  With scales per 128 channels the partial sums leave no registers
// for 128 rows: mean 16: 89.8, 91.5; 32: 121, 111; 128: 281, 227.
template <typename F>
static auto with_shape(const LinearParams &p, const ExpertsArgs &a, F &&f)
{
    const long mean = a.places / a.E;
    if (mean > 64 && p.act_per_token) return f(Shape<1, 4, 4, MIXLLM_PREFILL_WD_LARGE>{});
    if (mean > 16) return f(Shape<1, 4, 2, MIXLLM_PREFILL_WD_SMALL>{});
    return f(Shape<1, 4, 1, MIXLLM_PREFILL_WD_SMALL>{});
}

bool experts_tiled_covers(const LinearParams &p, const ExpertsArgs &a)
{
    return with_shape(p, a, [&](auto shape) { return blocks_of<decltype(shape)>(p, a) <= MAX_WORK_ITEMS / decltype(shape)::THREADS; });
}

int launch_experts_linear(const LinearParams &p, const ExpertsArgs &a, hipStream_t st)
{
    if (!experts_cover(p)) return (int)hipErrorInvalidValue;
    if (a.places == 0) return (int)hipSuccess;
    if (p.x) return launch_experts_stream(p, a, st);
    if (!experts_tiled_covers(p, a)) return (int)hipErrorInvalidValue;
    return with_shape(p, a, [&](auto shape) { return launch_experts_shape<decltype(shape)>(p, a, st); });
}

int launch_experts_combine(int T, int k, int N, int places, const void *y, const float *weights, const int32_t *slots, const void *residual,
                           void *out, hipStream_t st)
{
    if (T == 0) return (int)hipSuccess;
    constexpr int MOST = 1 << 23;   // tokens of a launch: a block of 256 threads each
    auto go = [&](auto kernel, int v) {
        for (int t = 0; t < T; t += MOST) {
            const size_t cell = (size_t)t * N, choice = (size_t)t * k;
            hipLaunchKernelGGL(kernel, dim3(std::min(T - t, MOST), (N + 256 * v - 1) / (256 * v)), dim3(256), 0, st, std::min(T - t, MOST), k, N, places,
                               (const half_t *)y, weights + choice, slots + choice, residual ? (const half_t *)residual + cell : nullptr,
                               (half_t *)out + cell);
            if (hipError_t e = hipGetLastError()) return (int)e;
        }
        return (int)hipSuccess;
    };
    return N % 8 == 0 ? go(experts_combine_kernel<8>, 8) : go(experts_combine_kernel<1>, 1);
}

}  // namespace mixllm
