// The products of a mixture-of-experts layer: gate and up with the activation between, down with the sum over a token's
// experts.
#include "exchange.h"
#include "experts.h"
#include "skinny_kernel.h"

namespace gptq {
namespace moe {
namespace {

using skinny::NibbleMagic;
using skinny::as_half2;
using skinny::u32x4_t;
typedef float f32x2_t __attribute__((ext_vector_type(2)));

struct Args {
    const half_t *x;         // gate and up: [M, K], the tokens; down: [pairs, K], their activations
    const uint32_t *qweight; // [experts, K/8, N]
    const uint32_t *qzeros;
    const half_t *scales;
    const Grouping *grouping;
    const Unit *units;
    const int32_t *order;    // pairs by expert
    half_t *hidden;          // gate and up: [pairs, N/2]
    float *partial;          // down: [pairs, N]
    const int32_t *ids;      // down: [M, top_k]
    const float *weights;
    half_t *out;             // down: [M, N]
    unsigned *counters;      // down: one per column tile, zero between launches
    int M, top_k, K, N, group_size, experts;
};

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kCols = 64;  // of a workgroup; gate and up: 32 of each

// One workgroup: one unit (grid y) times 64 columns (grid x); its wavefronts split K.
template <int TM, bool DOWN>
__global__ __launch_bounds__(kThreads) void experts_kernel(const Args a)
{
    constexpr int ROWS = 16 * TM;
    __shared__ __align__(16) float red[kWaves][ROWS][kCols];
    __shared__ int s_last;
    const int units = a.grouping->units;
    const int u = blockIdx.y, tile = blockIdx.x;
    // (down: without any pair the first unit's workgroups still write the zeros)
    if (u >= units && !(DOWN && u == 0))
        return;
    const Unit unit = u < units ? a.units[u] : Unit{0, 0, 0, 0};
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cq = lane & 15, kg = lane >> 4;
    const int N = a.N, half_n = N / 2;

    if (unit.count > 0) {
        const int col = DOWN ? min(tile * kCols + 4 * cq, N - 4)
                             : cq < 8 ? tile * 32 + 4 * cq : half_n + tile * 32 + 4 * (cq - 8);
        const half_t *xrow[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int pair = a.order[unit.first + min(16 * i + cq, unit.count - 1)];
            xrow[i] = a.x + (size_t)(DOWN ? pair : pair / a.top_k) * a.K + kg * 8;
        }
        const size_t groups = a.K / a.group_size;
        const uint32_t *qweight = a.qweight + (size_t)unit.expert * (a.K / 8) * N + (size_t)kg * N + col;
        const uint32_t *qzeros = a.qzeros + (size_t)unit.expert * groups * (N / 8) + (col >> 3);
        const half_t *scales = a.scales + (size_t)unit.expert * groups * N + col;
        const int zshift = (col & 4) * 4;

        float4_t acc[TM][4];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                acc[i][t] = float4_t{0.f, 0.f, 0.f, 0.f};
        const NibbleMagic magic;
        const int steps = a.K / 32, per_wave = (steps + kWaves - 1) / kWaves;
        const int s0 = min(wave * per_wave, steps), s1 = min(s0 + per_wave, steps);
        for (int s = s0; s < s1; ++s) {
            const uint4 w = *reinterpret_cast<const uint4 *>(qweight + (size_t)s * 4 * N);
            const int g = s * 32 / a.group_size;
            const uint2 sc = *reinterpret_cast<const uint2 *>(scales + (size_t)g * N);
            const uint32_t zeros = qzeros[(size_t)g * (N / 8)] >> zshift;
            half8_t av[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) {  // the k order of the weights: halves (0,4) (1,5) (2,6) (3,7)
                const u32x4_t xv = *reinterpret_cast<const u32x4_t *>(xrow[i] + s * 32);
                const u32x4_t xp = {__builtin_amdgcn_perm(xv[2], xv[0], 0x05040100u),
                                    __builtin_amdgcn_perm(xv[2], xv[0], 0x07060302u),
                                    __builtin_amdgcn_perm(xv[3], xv[1], 0x05040100u),
                                    __builtin_amdgcn_perm(xv[3], xv[1], 0x07060302u)};
                av[i] = __builtin_bit_cast(half8_t, xp);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t word = t == 0 ? w.x : t == 1 ? w.y : t == 2 ? w.z : w.w;
                const uint32_t z = zeros >> (4 * t) & 15u, zz = z | z << 16;
                const half2_t neg_lo = as_half2(zz | 0xE400E400u), neg_hi = as_half2(zz << 4 | 0xD400D400u);
                const uint32_t pair = t < 2 ? sc.x : sc.y;
                const float sf = (float)__builtin_bit_cast(half_t, (uint16_t)(t & 1 ? pair >> 16 : pair & 0xffffu));
                const uint32_t w8 = word >> 8;
                const half2_t c0 = as_half2((word & magic.mask_lo) | magic.bias_lo) + neg_lo;
                const half2_t c1 = as_half2((word & magic.mask_hi) | magic.bias_hi) + neg_hi;
                const half2_t c2 = as_half2((w8 & magic.mask_lo) | magic.bias_lo) + neg_lo;
                const half2_t c3 = as_half2((w8 & magic.mask_hi) | magic.bias_hi) + neg_hi;
                const half8_t b = half8_t{c0[0], c0[1], c1[0], c1[1], c2[0], c2[1], c3[0], c3[1]};
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const float4_t d =
                        __builtin_amdgcn_mfma_f32_16x16x32_f16(av[i], b, float4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[i][t][r] = __builtin_fmaf(sf, d[r], acc[i][t][r]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<float4_t *>(&red[wave][16 * i + 4 * kg + r][4 * cq]) =
                    float4_t{acc[i][0][r], acc[i][1][r], acc[i][2][r], acc[i][3][r]};
    }
    __syncthreads();
    auto total = [&](int row, int c) {
        float4_t s = *reinterpret_cast<const float4_t *>(&red[0][row][c]);
#pragma unroll
        for (int w = 1; w < kWaves; ++w)
            s += *reinterpret_cast<const float4_t *>(&red[w][row][c]);
        return s;
    };
    if (!DOWN) {
        for (int e = tid; e < unit.count * 8; e += kThreads) {
            const int row = e / 8, c = e % 8 * 4;
            const float4_t gate = total(row, c), up = total(row, 32 + c);
            half4_t h;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                h[j] = (half_t)(gate[j] / (1.f + __expf(-gate[j])) * up[j]);
            const int pair = a.order[unit.first + row];
            *reinterpret_cast<half4_t *>(a.hidden + (size_t)pair * half_n + tile * 32 + c) = h;
        }
        return;
    }
    for (int e = tid; e < unit.count * 16; e += kThreads) {
        const int row = e / 16, c = e % 16 * 4, n = tile * kCols + c;
        if (n >= N)
            continue;
        const float4_t s = total(row, c);
        unsigned long long *dst =
            reinterpret_cast<unsigned long long *>(a.partial + (size_t)a.order[unit.first + row] * N + n);
        __hip_atomic_store(dst, __builtin_bit_cast(unsigned long long, f32x2_t{s[0], s[1]}), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(dst + 1, __builtin_bit_cast(unsigned long long, f32x2_t{s[2], s[3]}), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
    }
    // the last unit of this column tile to arrive adds every token's experts, in the order of their places (exchange.h)
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (tid == 0)
        s_last = slice_arrive(a.counters + tile) == (unsigned)(max(units, 1) - 1);
    __syncthreads();
    if (!s_last)
        return;
    slice_acquire();
    for (int e = tid; e < a.M * 16; e += kThreads) {
        const int m = e / 16, n = tile * kCols + e % 16 * 4;
        if (n >= N)
            continue;
        float4_t s = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < a.top_k; ++j) {
            const int id = a.ids[m * a.top_k + j];
            if (id < 0 || id >= a.experts)
                continue;
            const float w = a.weights[m * a.top_k + j];
            const unsigned long long *src =
                reinterpret_cast<const unsigned long long *>(a.partial + (size_t)(m * a.top_k + j) * N + n);
            const f32x2_t lo = __builtin_bit_cast(f32x2_t, __hip_atomic_load(src, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
            const f32x2_t hi =
                __builtin_bit_cast(f32x2_t, __hip_atomic_load(src + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
            s[0] = __builtin_fmaf(w, lo[0], s[0]);
            s[1] = __builtin_fmaf(w, lo[1], s[1]);
            s[2] = __builtin_fmaf(w, hi[0], s[2]);
            s[3] = __builtin_fmaf(w, hi[1], s[3]);
        }
        *reinterpret_cast<half4_t *>(a.out + (size_t)m * N + n) =
            half4_t{(half_t)s[0], (half_t)s[1], (half_t)s[2], (half_t)s[3]};
    }
    if (tid == 0)
        __hip_atomic_store(a.counters + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

size_t align256(size_t v)
{
    return (v + 255) & ~(size_t)255;
}

}  // namespace

int unit_rows(int M, int experts, int top_k)
{
    return M > 16 && M * top_k > 8 * experts ? 32 : 16;
}

Layout make_layout(int M, int hidden, int inter, int experts, int top_k)
{
    const size_t pairs = (size_t)M * top_k;
    Layout l;
    l.grouping = 0;
    l.units = 256;
    l.pairs = align256(l.units + sizeof(Unit) * max_units((int)pairs, experts, unit_rows(M, experts, top_k)));
    l.ids = align256(l.pairs + 4 * pairs);
    l.weights = align256(l.ids + 4 * pairs);
    l.hidden = align256(l.weights + 4 * pairs);
    l.partial = align256(l.hidden + sizeof(half_t) * pairs * inter);
    l.bytes = align256(l.partial + sizeof(float) * pairs * hidden);
    return l;
}

hipError_t launch_experts(const Call &c, const Layout &l, unsigned char *scratch, unsigned *counters, hipStream_t stream)
{
    const int rows = unit_rows(c.M, c.experts, c.top_k), pairs = c.M * c.top_k;
    Grouping *grouping = reinterpret_cast<Grouping *>(scratch + l.grouping);
    Unit *units = reinterpret_cast<Unit *>(scratch + l.units);
    int32_t *order = reinterpret_cast<int32_t *>(scratch + l.pairs);
    const hipError_t err = launch_group(c.ids, pairs, c.experts, rows, grouping, units, order, stream);
    if (err != hipSuccess)
        return err;
    Args a = {};
    a.x = c.x;
    a.qweight = c.gate_up_qweight;
    a.qzeros = c.gate_up_qzeros;
    a.scales = c.gate_up_scales;
    a.grouping = grouping;
    a.units = units;
    a.order = order;
    a.hidden = reinterpret_cast<half_t *>(scratch + l.hidden);
    a.partial = reinterpret_cast<float *>(scratch + l.partial);
    a.ids = c.ids;
    a.weights = c.weights;
    a.out = c.out;
    a.counters = counters;
    a.M = c.M;
    a.top_k = c.top_k;
    a.K = c.hidden;
    a.N = 2 * c.inter;
    a.group_size = c.group_size;
    a.experts = c.experts;
    const int most = max_units(pairs, c.experts, rows);
    const dim3 grid0(c.inter / 32, most), grid1((c.hidden + kCols - 1) / kCols, most);
    if (rows == 16)
        experts_kernel<1, false><<<grid0, kThreads, 0, stream>>>(a);
    else
        experts_kernel<2, false><<<grid0, kThreads, 0, stream>>>(a);
    a.x = a.hidden;
    a.qweight = c.down_qweight;
    a.qzeros = c.down_qzeros;
    a.scales = c.down_scales;
    a.K = c.inter;
    a.N = c.hidden;
    if (rows == 16)
        experts_kernel<1, true><<<grid1, kThreads, 0, stream>>>(a);
    else
        experts_kernel<2, true><<<grid1, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace moe
}  // namespace gptq
