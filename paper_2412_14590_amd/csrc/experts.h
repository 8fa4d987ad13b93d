// Which tile of which expert a block takes, found on the device: how many rows an expert has is known there only.
#pragma once

#include "internal.h"

namespace mixllm {

// inclusive sum over the lanes of a wave (all active), inside rows of 16 lanes, then over the rows: six additions
template <int CTRL, int ROWS>
static __device__ inline int add_dpp(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
static __device__ inline int wave_scan(int v)
{
    v = add_dpp<0x111, 0xf>(v);   // row_shr:1, 2, 4, 8
    v = add_dpp<0x112, 0xf>(v);
    v = add_dpp<0x114, 0xf>(v);
    v = add_dpp<0x118, 0xf>(v);
    v = add_dpp<0x142, 0xa>(v);   // row_bcast:15 into rows 1 and 3
    return add_dpp<0x143, 0xc>(v);   // row_bcast:31 into rows 2 and 3
}
static __device__ inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// first place and rows of expert e, clamped to the places there are
static __device__ inline void clamp_rows(const ExpertsArgs &a, int lo, int hi, int &first, int &count)
{
    first = min(max(lo, 0), a.places);
    count = max(min(hi, a.places) - first, 0);
}
static __device__ inline void expert_rows(const ExpertsArgs &a, int e, int &first, int &count) { clamp_rows(a, a.offsets[e], a.offsets[e + 1], first, count); }

// The same and its entry of the table for an expert that is the same for the whole wave: by scalar loads, which come back
// past the hand-issued vector loads in flight (nothing writes either array while the kernels of the experts run).
template <typename T>
using constant_t = const __attribute__((address_space(4))) T;
static __device__ inline void expert_rows_uniform(const ExpertsArgs &a, int e, int &first, int &count)
{
    constant_t<int32_t> *o = (constant_t<int32_t> *)a.offsets;
    e = uniform(e);
    clamp_rows(a, o[e], o[e + 1], first, count);
}
static __device__ inline ExpertEntry expert_entry(const ExpertsArgs &a, int e)
{
    constant_t<ExpertEntry> *t = (constant_t<ExpertEntry> *)a.table + uniform(e);
    return ExpertEntry{t->w4, t->w8, t->s4, t->s8, t->z4, t->perm, t->n8, t->n4, t->ntiles8, t->ntiles4};
}

// Row `m` of an expert's (or the batch's) rows as a row of the activations: itself, or through the route's list
template <bool ROWS>
static __device__ inline int token_row(const LinearParams &p, int m)
{
    if constexpr (ROWS) return p.rows ? (int)min((unsigned)p.rows[m] / (unsigned)p.rows_per_token, (unsigned)(p.tokens - 1)) : m;   // (-1 too)
    return m;
}

}  // namespace mixllm
