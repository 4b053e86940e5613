// Routing of tokens to experts, and the grouping of (token, expert) pairs by expert.
#include "experts.h"
#include "wave_ops.h"

namespace gptq {
namespace moe {
namespace {

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

constexpr int kRouteWaves = 4;

template <int PER_LANE, typename T>
__global__ __launch_bounds__(64 * kRouteWaves) void route_kernel(const T *logits, int32_t *ids, float *weights, int M,
                                                                 int experts, int top_k, int renormalize)
{
    const int lane = threadIdx.x & 63;
    const int m = blockIdx.x * kRouteWaves + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (m >= M)
        return;
    int id;
    float weight;
    route_token<PER_LANE>(logits + (size_t)m * experts, experts, top_k, renormalize != 0, lane, id, weight);
    if (lane < top_k) {
        ids[(size_t)m * top_k + lane] = id;
        weights[(size_t)m * top_k + lane] = weight;
    }
}

template <typename T>
hipError_t route(const T *logits, int32_t *ids, float *weights, int M, int experts, int top_k, int renormalize,
                 hipStream_t stream)
{
    const dim3 grid((M + kRouteWaves - 1) / kRouteWaves), block(64 * kRouteWaves);
    if (experts <= 64)
        route_kernel<1><<<grid, block, 0, stream>>>(logits, ids, weights, M, experts, top_k, renormalize);
    else if (experts <= 256)
        route_kernel<4><<<grid, block, 0, stream>>>(logits, ids, weights, M, experts, top_k, renormalize);
    else
        route_kernel<16><<<grid, block, 0, stream>>>(logits, ids, weights, M, experts, top_k, renormalize);
    return hipGetLastError();
}

// One workgroup groups all pairs: a count per expert, an exclusive sum over the experts of pairs and of units, then every
// pair takes the next place of its expert.  Which place a pair gets depends on the order of LDS atomics, but nothing that is
// computed from it does: a row's result does not depend on the rows beside it, and is kept under its pair.
constexpr int kGroupThreads = 1024;
static_assert(kGroupThreads >= kMaxExperts, "a thread per expert");

__global__ __launch_bounds__(kGroupThreads) void group_kernel(const int32_t *ids, int pairs, int experts, int rows,
                                                              Grouping *grouping, Unit *units, int32_t *order)
{
    __shared__ int count[kMaxExperts], next[kMaxExperts];
    __shared__ int wave_pairs[kGroupThreads / 64], wave_units[kGroupThreads / 64];
    const int tid = threadIdx.x;
    count[tid] = 0;
    __syncthreads();
    for (int p = tid; p < pairs; p += kGroupThreads) {
        const int e = ids[p];
        if (e >= 0 && e < experts)
            atomicAdd(&count[e], 1);
    }
    __syncthreads();
    const int lane = tid & 63, wave = tid >> 6;
    const int mine = count[tid], my_units = (mine + rows - 1) / rows;
    int sum_pairs = mine, sum_units = my_units;  // inclusive, over the wavefront
    for (int d = 1; d < 64; d <<= 1) {
        const int a = __shfl_up(sum_pairs, d), b = __shfl_up(sum_units, d);
        if (lane >= d) {
            sum_pairs += a;
            sum_units += b;
        }
    }
    if (lane == 63) {
        wave_pairs[wave] = sum_pairs;
        wave_units[wave] = sum_units;
    }
    __syncthreads();
    int first = sum_pairs - mine, unit = sum_units - my_units;
    for (int w = 0; w < wave; ++w) {
        first += wave_pairs[w];
        unit += wave_units[w];
    }
    next[tid] = first;
    for (int u = 0; u < my_units; ++u)
        units[unit + u] = Unit{tid, first + u * rows, min(rows, mine - u * rows), 0};
    if (tid == kGroupThreads - 1)
        grouping->units = unit + my_units;
    __syncthreads();
    for (int p = tid; p < pairs; p += kGroupThreads) {
        const int e = ids[p];
        if (e >= 0 && e < experts)
            order[atomicAdd(&next[e], 1)] = p;
    }
}

}  // namespace

hipError_t launch_route(const void *logits, bool fp32, int32_t *ids, float *weights, int M, int experts, int top_k,
                        bool renormalize, hipStream_t stream)
{
    if (fp32)
        return route(static_cast<const float *>(logits), ids, weights, M, experts, top_k, renormalize, stream);
    return route(static_cast<const half_t *>(logits), ids, weights, M, experts, top_k, renormalize, stream);
}

hipError_t launch_group(const int32_t *ids, int pairs, int experts, int rows, Grouping *grouping, Unit *units,
                        int32_t *order, hipStream_t stream)
{
    group_kernel<<<1, kGroupThreads, 0, stream>>>(ids, pairs, experts, rows, grouping, units, order);
    return hipGetLastError();
}

}  // namespace moe
}  // namespace gptq
