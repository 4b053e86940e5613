// Routing of one token by one wavefront.
#pragma once

#include "kernels.h"
#include "wave_ops.h"

namespace gptq {
namespace moe {

// Logits as unsigned integers of the same order; 0 for those that are masked (-infinity, NaN).  Adding zero makes equal
// logits equal bits: -0.0 becomes +0.0.
__device__ __forceinline__ uint32_t order_of(float v)
{
    const uint32_t bits = __builtin_bit_cast(uint32_t, v + 0.f);
    const uint32_t key = bits & 0x80000000u ? ~bits : bits | 0x80000000u;
    return v > -__builtin_inff() ? key : 0u;  // (false for NaN)
}

__device__ __forceinline__ float logit_of(uint32_t key)
{
    return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// exp(v - top) of unmasked logits; infinities among themselves are equal.
__device__ __forceinline__ float share_of(uint32_t key, uint32_t top)
{
    return key == 0 ? 0.f : key == top ? 1.f : expf(logit_of(key) - logit_of(top));
}

// One wavefront routes one token: lane l holds experts l, l + 64, ... as ordered integers; every place is a maximum over
// the wavefront and a search for the first expert that has it, lowest index first.
template <int PER_LANE, typename T>
__device__ __forceinline__ void route_token(const T *logits, int experts, int top_k, bool renormalize, int lane, int &id,
                                            float &weight)
{
    uint32_t key[PER_LANE];
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < PER_LANE; ++i) {
        const int e = lane + 64 * i;
        key[i] = e < experts ? order_of((float)logits[e]) : 0u;
        mine = key[i] > mine ? key[i] : mine;
    }
    const uint32_t top = wave_max(mine);
    float total = 0.f;
    if (!renormalize) {
#pragma unroll
        for (int i = 0; i < PER_LANE; ++i)
            total += share_of(key[i], top);
        total = wave_sum(total);
    }
    uint32_t chosen = 0;
    id = -1;
    uint32_t best = top;
    for (int j = 0; j < top_k && best != 0; ++j) {  // (uniform: `best` is the wavefront's)
        int e = -1;
#pragma unroll
        for (int i = 0; i < PER_LANE; ++i) {
            const uint64_t have = __ballot(key[i] == best);
            if (e < 0 && have) {
                const int l = __builtin_ctzll(have);
                e = l + 64 * i;
                key[i] = lane == l ? 0u : key[i];
            }
        }
        if (lane == j) {
            id = e;
            chosen = best;
        }
        mine = 0;
#pragma unroll
        for (int i = 0; i < PER_LANE; ++i)
            mine = key[i] > mine ? key[i] : mine;
        best = wave_max(mine);
    }
    const float share = share_of(chosen, top);
    if (renormalize)
        total = wave_sum(share);
    weight = chosen ? share / total : 0.f;
}

template <typename T>
__device__ __forceinline__ void route_any(const T *logits, int experts, int top_k, bool renormalize, int lane, int &id,
                                          float &weight)
{
    if (experts <= 64)
        route_token<1>(logits, experts, top_k, renormalize, lane, id, weight);
    else if (experts <= 256)
        route_token<4>(logits, experts, top_k, renormalize, lane, id, weight);
    else
        route_token<16>(logits, experts, top_k, renormalize, lane, id, weight);
}

}  // namespace moe
}  // namespace gptq
