// What follows the product in a block, on the fp32 sums while they are in registers: bias, activation or gate,
// residual; one rounding to fp16 at the end.  Shared by every kernel of the linear with an epilogue.
//
//   v = sum + bias[channel];   y = act(v) + residual        or, gated,   y = act(v[2 i]) v[2 i + 1] + residual
//
// Gated, channels 2 i and 2 i + 1 are gate and up of output i.  Where the list of 8-bit channels holds both of a pair or
// neither, a pair is two neighbouring rows of one packed part, starting at an even one: two neighbouring lanes of every
// kernel's output.  Each lane then finishes half of the pair's rows - the even lane the even ones, for which it
// needs the other's up values, the odd lane the odd ones, for which it needs the gates - so that one exchange
// between neighbours (a vector instruction) serves two rows and no lane idles in the exponential.
//
// It costs what it stores less: K = 1408, N = 4096, 16384 rows 143.1 us without and 141.5 with an empty epilogue, K = 4096, N = 2816 gated with
// silu 234 and 241; a pass of its own over those sums would read and write 138 MB, 28 us.
#pragma once

#include <type_traits>

#include "internal.h"

namespace mixllm {

// x / (1 + exp(-t)): the hardware's exponential and reciprocal are good to 1 ulp, the exponent's rounding to |t| 2^-24
// relative, three decimal places below the fp16 result's own.  A large -t gives x / inf = 0.
static __device__ inline float times_sigmoid(float x, float t) { return x * __builtin_amdgcn_rcpf(1.0f + __expf(-t)); }

template <int ACT>
static __device__ inline float activation(float v)
{
    if constexpr (ACT == MIXLLM_ACT_RELU) return v < 0.0f ? 0.0f : v;   // (a NaN stays)
    if constexpr (ACT == MIXLLM_ACT_SILU) return times_sigmoid(v, v);
    // (the complement keeps its relative precision where the sum 1 + erf would cancel)
    if constexpr (ACT == MIXLLM_ACT_GELU) return 0.5f * v * erfcf(-0.70710678118654752f * v);
    // (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u))
    if constexpr (ACT == MIXLLM_ACT_GELU_TANH) return times_sigmoid(v, 1.5957691216057308f * (v + 0.044715f * v * v * v));
    return v;
}
// f(std::integral_constant<int, act>{}): one uniform branch around a loop over values, not one in it
template <typename F>
static __device__ __forceinline__ void with_activation(int act, F &&f)
{
    switch (act) {
    case MIXLLM_ACT_RELU: f(std::integral_constant<int, MIXLLM_ACT_RELU>{}); break;
    case MIXLLM_ACT_SILU: f(std::integral_constant<int, MIXLLM_ACT_SILU>{}); break;
    case MIXLLM_ACT_GELU: f(std::integral_constant<int, MIXLLM_ACT_GELU>{}); break;
    case MIXLLM_ACT_GELU_TANH: f(std::integral_constant<int, MIXLLM_ACT_GELU_TANH>{}); break;
    default: f(std::integral_constant<int, MIXLLM_ACT_NONE>{}); break;
    }
}

// the value of the neighbouring lane (0 <-> 1, 2 <-> 3, ...); both lanes are active
static __device__ inline float of_neighbour(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0xB1, 0xf, 0xf, true)); }

// Values of two consecutive rows in a pair of lanes -> this lane's gate and up (the even lane takes the first row)
static __device__ inline void exchange_pair(float row0, float row1, bool odd, float &gate, float &up)
{
    const float got = of_neighbour(odd ? row0 : row1);
    gate = odd ? got : row0;
    up = odd ? row1 : got;
}

// One channel's sums (already scaled) of R consecutive rows from m0 on, R = 1 or even, to the output.  ch = -1: none;
// every lane of the wave calls it.  Rows from p.M on are not stored.
template <int R>
static __device__ __forceinline__ void store_rows(const LinearParams &p, float (&v)[R], int m0, int ch)
{
    const EpilogueArgs &e = p.ep;
    asm volatile("" : "+v"(m0), "+v"(ch));   // (no address of the output is computed, and kept in registers, before the K loop)
    const int c = max(ch, 0);
    // (every branch runs to its stores: values that come together behind a branch would be copied from register to register)
    const float b = e.bias ? (float)e.bias[c] : 0.0f;
    auto finish = [&](auto gated, auto act) {
        constexpr bool GATED = decltype(gated)::value, PAIR = GATED && R > 1;
        constexpr int ACT = decltype(act)::value, O = PAIR ? R / 2 : R, STEP = PAIR ? 2 : 1;   // rows this lane finishes
        const bool odd = threadIdx.x & 1;
        const int first = PAIR ? m0 + (odd ? 1 : 0) : m0, stride = GATED ? p.N / 2 : p.N, col = GATED ? c >> 1 : c;
        half_t r[O];
#pragma unroll
        for (int i = 0; i < O; ++i) r[i] = e.residual ? e.residual[(size_t)min(first + i * STEP, p.M - 1) * stride + col] : (half_t)0.0f;
        float out[O];
#pragma unroll
        for (int i = 0; i < O; ++i) {
            if constexpr (PAIR) {
                float gate, up;
                exchange_pair(v[2 * i] + b, v[2 * i + 1] + b, odd, gate, up);
                out[i] = activation<ACT>(gate) * up;
            } else if constexpr (GATED) {
                const float up = of_neighbour(v[i] + b);   // (the odd lane's result is not stored)
                out[i] = activation<ACT>(v[i] + b) * up;
            } else
                out[i] = activation<ACT>(v[i] + b);
        }
        const bool stores = ch >= 0 && !(GATED && !PAIR && odd);
#pragma unroll
        for (int i = 0; i < O; ++i)
            if (stores && first + i * STEP < p.M) p.y[(size_t)(first + i * STEP) * stride + col] = (half_t)(out[i] + (float)r[i]);
    };
    if (e.gated) with_activation(e.act, [&](auto act) { finish(std::true_type{}, act); });
    else with_activation(e.act, [&](auto act) { finish(std::false_type{}, act); });
}

}  // namespace mixllm
