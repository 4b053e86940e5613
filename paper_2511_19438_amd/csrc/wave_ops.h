// Reductions over a wavefront of 64 lanes with data-parallel primitives (no LDS), gfx9.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gptq {

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_zero(uint32_t v)  // lanes without a source get 0
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}

// Combines in a fixed order; the result (the same in every lane) is what lane 63 gathers.  0 is neutral for both uses.
template <typename OP>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, OP op)
{
    v = op(v, dpp_or_zero<0x111, 0xf>(v));  // row_shr:1, 2, 4, 8: lane 15 of every row of 16 has its row
    v = op(v, dpp_or_zero<0x112, 0xf>(v));
    v = op(v, dpp_or_zero<0x114, 0xf>(v));
    v = op(v, dpp_or_zero<0x118, 0xf>(v));
    v = op(v, dpp_or_zero<0x142, 0xa>(v));  // row_bcast:15 into rows 1 and 3
    v = op(v, dpp_or_zero<0x143, 0xc>(v));  // row_bcast:31 into rows 2 and 3
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    return wave_reduce(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

__device__ __forceinline__ float wave_sum(float v)
{
    return __builtin_bit_cast(float, wave_reduce(__builtin_bit_cast(uint32_t, v), [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
    }));
}

}  // namespace gptq
