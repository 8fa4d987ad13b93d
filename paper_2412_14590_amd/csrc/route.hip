// Router of a layer of experts: scores, a bias for balance, groups of experts, top-k, weights, and the lists of
// rows per expert that the experts' products read.
//
// A token's experts are spread over LANES lanes, SLOTS consecutive experts a lane: a wave for every token, or, where
// there are tokens enough, 16 lanes, whose maxima are rotations inside a row of lanes (an instruction
// each) that serve four tokens at once.  The k experts are found one after the other: the largest key, then the smallest
// index that has it, so that ties go to the lowest index.  Keys are the logits themselves where score and choice have the
// same order (no bias, no sum of two scores), which is exact; otherwise score + bias in 64 bits, because two experts whose
// 32-bit scores round alike are in earnest in one batch of a few thousand tokens, and the choice would hang on the rounding
// of an exponential.
//
// The lists: a token takes an expert at most once, so the tokens of a group of 64 that took expert e are the bits of
// one 64-bit word in LDS (an OR is the same in any order), the rank of an assignment among its expert's is a count of
// the bits below its own, and the sorted order is that of the assignments' numbers without a sort.  Up to 16 tokens
// one block does it all in one launch; beyond, the first launch leaves the counts of every block and expert, and the
// second adds up those of the blocks before its own.
//
// Bound by instructions and latency, not by the logits' few bytes: one token of 64 experts 3.6 us (one launch after the other in a graph; a
// call from Python takes the host 6.3 to 7.4, five result tensors among it), 61 tokens of 256 in groups 12.3, 16384 tokens of
// 128 experts, 4 MB of logits, 16 (10 and 6 of the two launches).
#include <algorithm>
#include <type_traits>

#include "internal.h"

namespace mixllm {

namespace {

constexpr int THREADS = 1024;
constexpr int MAX_BLOCKS = 256;   // blocks that the tokens are cut into for counting (a block of the lists reads the counts of all)
// Tokens up to which one block takes a wave for each (us, one launch and two: 64 experts, 4 of them: 1 token 3.8 and 6.8, 16 tokens 6.2 and 7.5,
// 32 tokens 8.3 and 7.6; 256 experts, 8 of them: 1 token 5.2 and 8.0, 16 tokens 8.8 and 8.8)
constexpr int ONE_LAUNCH = 16;
constexpr size_t LDS_CELLS = 140 * 1024;   // LDS for the keys of the waves' tokens, where groups are chosen
// threads of a block of route_kernel: sixteen 64-bit keys a lane take more than the 128 registers of a block of 1024
constexpr int threads_of(int slots, bool wide) { return slots == 16 && wide ? 512 : THREADS; }

template <int CTRL>
__device__ inline float dpp(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true)); }
template <int CTRL>
__device__ inline int dpp(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ inline double dpp(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = (uint32_t)dpp<CTRL>((int)(uint32_t)b), hi = (uint32_t)dpp<CTRL>((int)(uint32_t)(b >> 32));
    return __builtin_bit_cast(double, lo | (hi << 32));
}
__device__ inline float at_lane(float v, int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); }
__device__ inline int at_lane(int v, int l) { return __builtin_amdgcn_readlane(v, l); }
__device__ inline double at_lane(double v, int l)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = (uint32_t)at_lane((int)(uint32_t)b, l), hi = (uint32_t)at_lane((int)(uint32_t)(b >> 32), l);
    return __builtin_bit_cast(double, lo | (hi << 32));
}
// op over the LANES lanes of a token; every lane gets the result (all lanes of the wave are active)
template <int LANES, typename T, typename F>
__device__ inline T over_token(T v, F &&op)
{
    v = op(v, dpp<0x121>(v));   // row_ror:1, 2, 4, 8
    v = op(v, dpp<0x122>(v));
    v = op(v, dpp<0x124>(v));
    v = op(v, dpp<0x128>(v));
    if constexpr (LANES == 64) v = op(op(at_lane(v, 0), at_lane(v, 16)), op(at_lane(v, 32), at_lane(v, 48)));
    return v;
}
struct Max {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
    __device__ double operator()(double a, double b) const { return fmax(a, b); }
    __device__ int operator()(int a, int b) const { return max(a, b); }
};
struct Min {
    __device__ int operator()(int a, int b) const { return min(a, b); }
};
struct Sum {
    template <typename T>
    __device__ T operator()(T a, T b) const { return a + b; }
};

constexpr int LOWEST_BITS = (int)0xff800000u;
__device__ inline float lowest() { return __builtin_bit_cast(float, LOWEST_BITS); }

// Keys: scores in 64 bits, or the logits as whole numbers in the same order (a maximum of floats costs an instruction more
// per operand, to quiet what might be a signalling NaN).
template <bool WIDE>
struct KeyOf {
    using type = int;
    static __device__ int none() { return (int)0x80000000u; }   // below any logit's
    static __device__ int of(float l)
    {
        const int b = __builtin_bit_cast(int, l + 0.0f);   // (one zero)
        return l > lowest() ? b ^ ((b >> 31) & 0x7fffffff) : none();
    }
    static __device__ float logit(int k) { return __builtin_bit_cast(float, k ^ ((k >> 31) & 0x7fffffff)); }
    static __device__ double wide(int k) { return k == none() ? -HUGE_VAL : (double)logit(k); }
};
template <>
struct KeyOf<true> {
    using type = double;
    static __device__ double none() { return -HUGE_VAL; }
    static __device__ double wide(double k) { return k; }
};

// One wave's tokens: 64 / LANES of them, from `t0` on; those from `t_end` on are none.  `cells`: this wave's LDS
// (groups only): [token][E] keys and [token][groups] scores of groups.  Leaves ids and weights in memory and the
// tokens' bits (counted from `t_base`) in `taken`.
template <int LANES, int SLOTS, bool WIDE>
__device__ inline void route_tokens(const RouteParams &p, int t0, int t_end, int t_base, double *cells, unsigned long long *taken)
{
    using KEY = KeyOf<WIDE>;
    using Key = typename KEY::type;
    const int lane = threadIdx.x & 63, sub = lane % LANES, in_wave = lane / LANES;
    const int tok = t0 + in_wave;
    const bool live = tok < t_end;
    const int row = min(tok, t_end - 1);
    const bool on = !p.mask || p.mask[row] != 0;
    float l[SLOTS];
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
        const int e = sub * SLOTS + s;
        float v = lowest();
        if (e < p.E) v = p.half ? (float)((const half_t *)p.logits)[(size_t)row * p.ld + e] : ((const float *)p.logits)[(size_t)row * p.ld + e];
        l[s] = on && v > lowest() ? v : lowest();   // (a NaN is not greater)
    }
    float m = l[0];
#pragma unroll
    for (int s = 1; s < SLOTS; ++s) m = fmaxf(m, l[s]);
    m = over_token<LANES>(m, Max{});
    // exp(l - m); the largest logits give 1 where they are infinite, too
    auto from_top = [&](float v) { return v == m ? 1.0 : exp((double)v - (double)m); };

    Key c[SLOTS];
    double total = 0.0;   // of a softmax over all experts, where it is needed
    if constexpr (WIDE) {
        if (!p.sigmoid) {
            double part = 0.0;
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) {
                c[s] = l[s] > lowest() ? from_top(l[s]) : 0.0;
                part += c[s];
            }
            total = over_token<LANES>(part, Sum{});
        }
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            double v = p.sigmoid ? 1.0 / (1.0 + exp(-(double)l[s])) : c[s] / total;
            if (p.bias) v += (double)p.bias[min(sub * SLOTS + s, p.E - 1)];
            c[s] = l[s] > lowest() && v > -HUGE_VAL ? v : -HUGE_VAL;
        }
    } else {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) c[s] = KEY::of(l[s]);
        // (Exponentials of all experts in 64 bits, so that a weight is rounded once, as everywhere: in 32 bits it was off by twice that.
        // 16384 tokens, us, renormalized, with the sum in 32 and in 64 bits: 64 experts 12.7, 12.9, 13.8; 128: 16.1, 17.0, 18.5.)
        if (!p.sigmoid && !p.renormalize) {
            double part = 0.0;
#pragma unroll
            for (int s = 0; s < SLOTS; ++s) part += l[s] > lowest() ? from_top(l[s]) : 0.0;
            total = over_token<LANES>(part, Sum{});
        }
    }

    if (p.groups > 1) {
        // The keys through LDS: `width` neighbouring lanes (a power of two) find the score of a group, its rank among the
        // groups, and take the group's experts out where it is not among the first.  (The wave's own cells: its LDS
        // accesses are in order, no barrier.)
        Key *mine = (Key *)cells + (size_t)in_wave * p.E;
        double *scores = cells + (size_t)(64 / LANES) * p.E + (size_t)in_wave * p.groups;
        const int size = p.E / p.groups;
        int width = 1;
        while (2 * width * p.groups <= LANES) width *= 2;
        const int part = sub & (width - 1), per_pass = LANES / width;   // groups at a time
#pragma unroll
        for (int s = 0; s < SLOTS; ++s)
            if (sub * SLOTS + s < p.E) mine[sub * SLOTS + s] = c[s];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int g0 = 0; g0 < p.groups; g0 += per_pass) {
            const int g = g0 + sub / width;
            double first = -HUGE_VAL, second = -HUGE_VAL;
            if (g < p.groups) {
#pragma unroll 4
                for (int i = part; i < size; i += width) {
                    const double v = KEY::wide(mine[g * size + i]);
                    second = fmax(second, fmin(first, v));
                    first = fmax(first, v);
                }
            }
            for (int d = 1; d < width; d *= 2) {
                const double f = __shfl_xor(first, d), o = __shfl_xor(second, d);
                second = fmax(fmax(second, o), fmin(first, f));
                first = fmax(first, f);
            }
            if (g < p.groups && part == 0) scores[g] = p.group_top2 && second > -HUGE_VAL ? first + second : first;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (int g0 = 0; g0 < p.groups; g0 += per_pass) {
            const int g = g0 + sub / width;
            const double own = scores[min(g, p.groups - 1)];
            int before = 0;
#pragma unroll 4
            for (int o = 0; o < p.groups; ++o) {
                const double v = scores[o];
                before += v > own || (v == own && o < g);
            }
            if (g < p.groups && before >= p.top_groups)
                for (int i = part; i < size; i += width) mine[g * size + i] = KEY::none();
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) c[s] = sub * SLOTS + s < p.E ? mine[sub * SLOTS + s] : KEY::none();
    }

    int my_id = -1;
    float my_logit = lowest();
    for (int j = 0; j < p.k; ++j) {
        Key best = c[0];
#pragma unroll
        for (int s = 1; s < SLOTS; ++s) best = Max{}(best, c[s]);
        const Key top = over_token<LANES>(best, Max{});
        int e_mine = 0x7fffffff;
#pragma unroll
        for (int s = SLOTS - 1; s >= 0; --s) e_mine = c[s] == top ? sub * SLOTS + s : e_mine;
        const int e = over_token<LANES>(e_mine, Min{});
        float logit = lowest();
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const bool taken = sub * SLOTS + s == e;
            if constexpr (WIDE) logit = taken ? l[s] : logit;
            c[s] = taken ? KEY::none() : c[s];
        }
        // its logit: the key itself, or the owner's
        if constexpr (WIDE) logit = over_token<LANES>(logit, Max{});
        else logit = KEY::logit(top);
        if (sub == j && top != KEY::none()) {
            my_id = e;
            my_logit = logit;
        }
    }

    double w = 0.0;
    if (my_id >= 0) w = p.sigmoid ? 1.0 / (1.0 + exp(-(double)my_logit)) : from_top(my_logit);
    if (p.renormalize) {
        const double sum = over_token<LANES>(w, Sum{});
        w = sum > 0.0 ? w / sum : 0.0;
    } else if (!p.sigmoid && my_id >= 0)
        w /= total;
    if (live && sub < p.k) {
        p.ids[(size_t)tok * p.k + sub] = my_id;
        p.weights[(size_t)tok * p.k + sub] = (float)(w * (double)p.scale);
        if (my_id >= 0) atomicOr(&taken[my_id], 1ull << (tok - t_base));
    }
}

// exclusive sums of n integers in LDS over all threads of the block, in place; returns the sum of all
__device__ inline int block_scan(int *v, int n, int *wave_sums)
{
    int before = 0;
    for (int i0 = 0; i0 < n; i0 += blockDim.x) {
        const int i = i0 + threadIdx.x;
        const int own = i < n ? v[i] : 0;
        int x = own;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int y = __shfl_up(x, d);
            if ((int)(threadIdx.x & 63) >= d) x += y;
        }
        if ((threadIdx.x & 63) == 63) wave_sums[threadIdx.x >> 6] = x;
        __syncthreads();
        int of_waves = 0, all = 0;
        for (int w = 0; w < (int)blockDim.x / 64; ++w) {
            if (w < (int)threadIdx.x >> 6) of_waves += wave_sums[w];
            all += wave_sums[w];
        }
        if (i < n) v[i] = before + of_waves + x - own;
        before += all;
        __syncthreads();
    }
    return before;
}

// row and slot of assignment `a`, which is expert e's (-1: none) and of the token `bit` of its 64; base[e]: place of the first of
// those 64 tokens' with expert e
__device__ inline void place(const RouteParams &p, int a, int e, int bit, const unsigned long long *taken, const int *base)
{
    int slot = -1;
    if (e >= 0) {
        slot = base[e] + __popcll(taken[e] & ((1ull << bit) - 1));
        p.rows[slot] = a;
    }
    p.slots[a] = slot;
}

// ONE: all tokens in one block, which makes the lists too.  Otherwise block b takes `span` tokens and leaves how many of
// them took each expert in counts[b].
template <int LANES, int SLOTS, bool WIDE, bool ONE>
__global__ __launch_bounds__(threads_of(SLOTS, WIDE)) void route_kernel(RouteParams p, int span)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    unsigned long long *taken = (unsigned long long *)smem;   // [E]
    int *count = (int *)(taken + p.E);                        // [E]
    int *wave_sums = count + p.E + (p.E & 1);                 // [16]
    constexpr int TPW = 64 / LANES;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    double *cells = (double *)(wave_sums + 16) + (size_t)wave * TPW * (p.E + p.groups);
    const int t_lo = blockIdx.x * span, t_hi = min(p.T, t_lo + span);
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
    for (int t = t_lo; t < t_hi; t += 64) {
        for (int e = threadIdx.x; e < p.E; e += blockDim.x) taken[e] = 0;
        __syncthreads();
        for (int u = t + wave * TPW; u < min(t + 64, t_hi); u += waves * TPW)
            route_tokens<LANES, SLOTS, WIDE>(p, u, min(t + 64, t_hi), t, cells, taken);
        __syncthreads();
        for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] += __popcll(taken[e]);
        if constexpr (!ONE) __syncthreads();
    }
    if constexpr (ONE) {
        __syncthreads();
        const int all = block_scan(count, p.E, wave_sums);
        for (int e = threadIdx.x; e < p.E; e += blockDim.x) p.offsets[e] = count[e];
        if (threadIdx.x == 0) p.offsets[p.E] = all;
        // (ids are read back from memory: written by this block, before the barriers of the scan)
        for (int i = threadIdx.x; i < p.T * p.k; i += blockDim.x) place(p, i, p.ids[i], i / p.k, taken, count);
        for (int i = all + threadIdx.x; i < p.T * p.k; i += blockDim.x) p.rows[i] = -1;
    } else {
        for (int e = threadIdx.x; e < p.Ep; e += blockDim.x) p.counts[(size_t)blockIdx.x * p.Ep + e] = e < p.E ? (uint16_t)count[e] : 0;
    }
}

// Block b makes the lists of `span` tokens (a multiple of 64): those of the blocks [b each, (b + 1) each) of the `nblocks`
// that counted.
__global__ __launch_bounds__(THREADS) void route_lists_kernel(RouteParams p, int span, int each, int nblocks)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    unsigned long long *taken = (unsigned long long *)smem;   // [E]
    int *base = (int *)(taken + p.E);                         // [E] all tokens' counts, then the offsets
    int *before = base + p.E;                                 // [E] counts of the tokens before this block's
    int *wave_sums = before + p.E;                            // [16]
    const int t_lo = blockIdx.x * span, t_hi = min(p.T, t_lo + span), own = blockIdx.x * each;
    // the first 64 tokens' ids are requested ahead of the counts (at most two a thread)
    const int n_first = (min(t_hi, t_lo + 64) - t_lo) * p.k;
    int first[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) first[i] = (int)threadIdx.x + i * THREADS < n_first ? p.ids[t_lo * p.k + threadIdx.x + i * THREADS] : -1;
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) {
        base[e] = before[e] = 0;
        taken[e] = 0;
    }
    __syncthreads();
    // a thread adds up eight experts of every `step`th block (whole numbers: any order)
    const int octets = p.Ep / 8, step = THREADS / octets, o = threadIdx.x % octets;
    if ((int)threadIdx.x / octets < step) {
        int sum[8] = {}, ahead[8] = {};
#pragma unroll 4
        for (int b = threadIdx.x / octets; b < nblocks; b += step) {
            const uint4 c = *(const uint4 *)(p.counts + (size_t)b * p.Ep + 8 * o);
            const uint32_t d[4] = {c.x, c.y, c.z, c.w};
            const bool is_ahead = b < own;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int n = (d[i >> 1] >> (16 * (i & 1))) & 0xffff;
                sum[i] += n;
                ahead[i] += is_ahead ? n : 0;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (8 * o + i < p.E) {
                if (sum[i]) atomicAdd(&base[8 * o + i], sum[i]);
                if (ahead[i]) atomicAdd(&before[8 * o + i], ahead[i]);
            }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (first[i] >= 0) atomicOr(&taken[first[i]], 1ull << (((int)threadIdx.x + i * THREADS) / p.k));
    __syncthreads();
    const int all = block_scan(base, p.E, wave_sums);
    if (blockIdx.x == 0) {
        for (int e = threadIdx.x; e < p.E; e += blockDim.x) p.offsets[e] = base[e];
        if (threadIdx.x == 0) p.offsets[p.E] = all;
    }
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) base[e] += before[e];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int at = (int)threadIdx.x + i * THREADS;
        if (at < n_first) place(p, t_lo * p.k + at, first[i], at / p.k, taken, base);
    }
    for (int t = t_lo + 64; t < t_hi; t += 64) {
        __syncthreads();
        for (int e = threadIdx.x; e < p.E; e += blockDim.x) {
            base[e] += __popcll(taken[e]);
            taken[e] = 0;
        }
        __syncthreads();
        const int n = (min(t_hi, t + 64) - t) * p.k;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int e = p.ids[t * p.k + i];
            if (e >= 0) atomicOr(&taken[e], 1ull << (i / p.k));
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += blockDim.x) place(p, t * p.k + i, p.ids[t * p.k + i], i / p.k, taken, base);
    }
    // places behind the last assignment
    for (long i = (long)t_lo * p.k + threadIdx.x; i < (long)t_hi * p.k; i += blockDim.x)
        if (i >= all) p.rows[i] = -1;
}

// Tokens of a block of the counting launch: a power of two from 4 on up to 64, then whole groups of 64; fewer than 2^16, so
// that a count fits 16 bits where all of them take one expert (2^24 tokens: a block more than MAX_BLOCKS)
int route_span(int T)
{
    int span = 4;
    while (span < 64 && (T + span - 1) / span > MAX_BLOCKS) span *= 2;
    return span < 64 ? span : 64 * std::min((T + 64 * MAX_BLOCKS - 1) / (64 * MAX_BLOCKS), 1023);
}

template <int LANES, int SLOTS>
int launch_lanes(const RouteParams &p, bool wide, hipStream_t st)
{
    constexpr int TPW = 64 / LANES;
    const bool one = p.T <= ONE_LAUNCH;
    const int span = one ? ONE_LAUNCH : route_span(p.T), blocks = one ? 1 : (p.T + span - 1) / span;
    // a wave for every TPW tokens, as many as a block holds; the lists want a few for the experts
    const size_t wave_cells = p.groups > 1 ? (size_t)TPW * (p.E + p.groups) * sizeof(double) : 0;
    int waves = (std::min(one ? std::max(p.T, 1) : span, 64) + TPW - 1) / TPW;
    if (one) waves = std::max(waves, std::min(4, (p.E + 63) / 64));
    waves = std::min(waves, threads_of(SLOTS, wide) / 64);
    if (wave_cells) waves = std::min(waves, (int)(LDS_CELLS / wave_cells));
    const size_t lds = (size_t)p.E * 8 + (size_t)(p.E + (p.E & 1)) * 4 + 64 + waves * wave_cells;
    auto go = [&](auto kernel) {
        if (lds > 48 * 1024)
            if (int e = ensure_dynamic_lds((const void *)kernel, lds)) return e;
        hipLaunchKernelGGL(kernel, dim3(blocks), dim3(64 * waves), lds, st, p, span);
        return (int)hipGetLastError();
    };
    if (one) {
        if constexpr (LANES == 64) return wide ? go(route_kernel<LANES, SLOTS, true, true>) : go(route_kernel<LANES, SLOTS, false, true>);
        return (int)hipErrorInvalidValue;
    }
    if (int e = wide ? go(route_kernel<LANES, SLOTS, true, false>) : go(route_kernel<LANES, SLOTS, false, false>)) return e;
    const int list_span = std::max(span, 64), lists = (p.T + list_span - 1) / list_span;
    hipLaunchKernelGGL(route_lists_kernel, dim3(lists), dim3(THREADS), (size_t)p.E * 16 + 64, st, p, list_span, list_span / span, blocks);
    return (int)hipGetLastError();
}

}  // namespace

size_t route_workspace_bytes(int T, int E)
{
    if (T <= ONE_LAUNCH) return 0;
    const int span = route_span(T);
    return (size_t)((T + span - 1) / span) * round_up(E, 8) * sizeof(uint16_t);
}

int launch_route(const RouteParams &p0, hipStream_t st)
{
    RouteParams p = p0;
    p.Ep = round_up(p.E, 8);
    // 64-bit keys wherever the order of the choice is not that of the logits
    const bool wide = p.bias || (p.groups > 1 && p.group_top2);
    // Four tokens a wave have fewer instructions a token, a wave for every token the shorter chain, and the more so the more
    // experts a lane of 16 holds.  us, a wave each and four a wave, 64 experts: 2048 tokens 10.8 and 10.4, 4096 12.2 and 10.4, 16384 20.1
    // and 12.8; 128 experts: 2048 11.0 and 11.2, 4096 12.8 and 11.6, 16384 24.8 and 17.0; 256 experts: 4096 14.5 and 14.5, 8192 19.5 and 18.1
    // (with a bias 28.8 and 24.6), 16384 28.9 and 23.7.
    const int slots = p.E <= 64 ? 4 : p.E <= 128 ? 8 : 16;
    if (p.T >= 2 * slots * cu_count() && p.E <= 256 && p.k <= 16) {
        if (slots == 4) return launch_lanes<16, 4>(p, wide, st);
        if (slots == 8) return launch_lanes<16, 8>(p, wide, st);
        return launch_lanes<16, 16>(p, wide, st);
    }
    if (p.E <= 64) return launch_lanes<64, 1>(p, wide, st);
    if (p.E <= 128) return launch_lanes<64, 2>(p, wide, st);
    if (p.E <= 256) return launch_lanes<64, 4>(p, wide, st);
    return launch_lanes<64, 16>(p, wide, st);
}

}  // namespace mixllm
