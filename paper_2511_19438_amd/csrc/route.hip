// Routing of tokens to experts, and the grouping of (token, expert) pairs by expert.
#include "experts.h"
#include "route_token.h"

namespace gptq {
namespace moe {
namespace {

constexpr int kRouteWaves = 4;

// A token to a wavefront, its logits dealt out to the lanes: top_k times the largest of all lanes, and one sum.  All in fp32.
// Bound by the launch and top_k dependent reductions over the lanes: one token of 8 experts 1.8 us, 2048 of 64 3.3 us.

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

// One workgroup groups all pairs: a count per expert, an exclusive sum of units over the experts, then every
// pair takes the next place of its expert.  Which place a pair gets depends on the order of LDS atomics, but nothing that is
// computed from it does: a row's result does not depend on the rows beside it, and is kept under its pair.
constexpr int kGroupThreads = 1024;
static_assert(kGroupThreads >= kMaxExperts, "a thread per expert");

__global__ __launch_bounds__(kGroupThreads) void group_kernel(const int32_t *ids, int pairs, int experts, int rows,
                                                              Grouping *grouping, Unit *units)
{
    __shared__ int count[kMaxExperts], first_unit[kMaxExperts];
    __shared__ int wave_units[kGroupThreads / 64];
    __shared__ int all;
    const int tid = threadIdx.x;
    count[tid] = 0;
    if (tid == 0)
        all = 0;
    __syncthreads();
    for (int p = tid; p < pairs; p += kGroupThreads) {
        const int e = ids[p];
        if (e >= 0 && e < experts)
            atomicAdd(&count[e], 1);
    }
    __syncthreads();
    const int lane = tid & 63, wave = tid >> 6;
    const int mine = count[tid], my_units = (mine + rows - 1) / rows;
    int unit = my_units;  // inclusive, over the wavefront
    for (int d = 1; d < 64; d <<= 1) {
        const int before = __shfl_up(unit, d);
        unit += lane >= d ? before : 0;
    }
    if (lane == 63)
        wave_units[wave] = unit;
    __syncthreads();
    unit -= my_units;
    for (int w = 0; w < wave; ++w)
        unit += wave_units[w];
    first_unit[tid] = unit;
    count[tid] = 0;
    for (int u = 0; u < my_units; ++u) {
        units[unit + u].expert = tid;
        units[unit + u].count = min(rows, mine - u * rows);
    }
    if (tid == kGroupThreads - 1)
        grouping->units = unit + my_units;
    if (mine > 0)
        atomicAdd(&all, mine);
    __syncthreads();
    for (int p = tid; p < pairs; p += kGroupThreads) {
        const int e = ids[p];
        if (e >= 0 && e < experts) {
            const int place = atomicAdd(&count[e], 1);
            units[first_unit[e] + place / rows].pairs[place % rows] = p;
        }
    }
    if (tid == 0)
        grouping->pairs = all;
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
                        hipStream_t stream)
{
    group_kernel<<<1, kGroupThreads, 0, stream>>>(ids, pairs, experts, rows, grouping, units);
    return hipGetLastError();
}

}  // namespace moe
}  // namespace gptq
