// Low-rank adapters of many requests: t = x A_l^T (shrink), out = base + s_l t B_l^T (expand), l the row's adapter.
//
// Both kernels take tiles of 16 rows and go through the different adapters of a tile, so that an adapter is read once for
// all of its rows there - a prompt's rows share one, a decode step's rows mostly have their own - and the host need not know
// which rows have which.  A row takes its values from its own adapter's product by selection: whatever another adapter
// holds, infinities included, does not reach it.
#include "adapters.h"

namespace gptq {
namespace lora {
namespace {

constexpr int kRows = 16;
constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

struct Args {
    const half_t *x, *a, *b, *base;
    const float *scaling;
    const int32_t *adapter;
    float *t;  // [slices, M, rank]
    half_t *out;
    long long ldx, ld_base, ld_out;
    int M, K, N, rank, adapters, slices, slice_steps;
};

// The adapters of a tile's rows: lane i < 16 has that of row i, -1 for none; `first` marks the lanes whose adapter no row
// before them has.
struct TileAdapters {
    int mine;
    uint32_t first;
    __device__ __forceinline__ TileAdapters(const Args &a, int m0, int lane)
    {
        mine = -1;
        if (lane < kRows && m0 + lane < a.M)
            mine = a.adapter[m0 + lane];
        if (mine < 0 || mine >= a.adapters)
            mine = -1;
        bool before = false;
#pragma unroll
        for (int j = 0; j < kRows; ++j)
            before |= j < lane && __builtin_amdgcn_readlane(mine, j) == mine;
        first = (uint32_t)__ballot(mine >= 0 && !before);
    }
};

constexpr int kRankTiles = 4;  // tiles of 16 ranks that are computed at a time

__global__ __launch_bounds__(kThreads) void shrink_kernel(const Args a)
{
    __shared__ float red[kWaves][kRows][16 * kRankTiles];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cq = lane & 15, kg = lane >> 4;
    const int m0 = blockIdx.x * kRows;
    const TileAdapters rows(a, m0, lane);
    const int steps = (a.K + 31) / 32;
    const int b0 = blockIdx.y * a.slice_steps, b1 = min(b0 + a.slice_steps, steps);
    const int per_wave = (b1 - b0 + kWaves - 1) / kWaves;
    const int s0 = min(b0 + wave * per_wave, b1), s1 = min(s0 + per_wave, b1);
    const half_t *x = a.x + min(m0 + cq, a.M - 1) * a.ldx;
    int index = 0;
    for (uint32_t left = rows.first; left != 0; left &= left - 1, ++index) {
        if (index % gridDim.z != blockIdx.z)
            continue;
        const int l = __builtin_amdgcn_readlane(rows.mine, __builtin_ctz(left));
        const half_t *la = a.a + (size_t)l * a.rank * a.K;
        for (int r0 = 0; r0 < a.rank; r0 += 16 * kRankTiles) {
            float4_t acc[kRankTiles];
            const half_t *arow[kRankTiles];
#pragma unroll
            for (int t = 0; t < kRankTiles; ++t) {
                acc[t] = float4_t{0.f, 0.f, 0.f, 0.f};
                arow[t] = la + (size_t)min(r0 + 16 * t + cq, a.rank - 1) * a.K;
            }
            for (int s = s0; s < s1; ++s) {
                const int k = s * 32 + kg * 8;
                half8_t xv = {}, av[kRankTiles] = {};
                if (k < a.K) {
                    xv = *reinterpret_cast<const half8_t *>(x + k);
#pragma unroll
                    for (int t = 0; t < kRankTiles; ++t)
                        if (r0 + 16 * t < a.rank)
                            av[t] = *reinterpret_cast<const half8_t *>(arow[t] + k);
                }
#pragma unroll
                for (int t = 0; t < kRankTiles; ++t)
                    if (r0 + 16 * t < a.rank)
                        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(xv, av[t], acc[t], 0, 0, 0);
            }
            __syncthreads();  // (the sums of the adapter or ranks before have been read)
#pragma unroll
            for (int t = 0; t < kRankTiles; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    red[wave][4 * kg + r][16 * t + cq] = acc[t][r];
            __syncthreads();
            for (int e = tid; e < kRows * 16 * kRankTiles; e += kThreads) {
                const int row = e / (16 * kRankTiles), c = e % (16 * kRankTiles);
                const int owner = __shfl(rows.mine, row);  // (a wavefront's 64 elements are one row: all lanes take part)
                if (owner != l || r0 + c >= a.rank)
                    continue;
                float sum = red[0][row][c];
#pragma unroll
                for (int w = 1; w < kWaves; ++w)
                    sum += red[w][row][c];
                a.t[((size_t)blockIdx.y * a.M + m0 + row) * a.rank + r0 + c] = sum;
            }
        }
    }
}

constexpr int kCols = 16 * kWaves;

__global__ __launch_bounds__(kThreads) void expand_kernel(const Args a)
{
    __shared__ __align__(16) float ts[kRows][kMaxRank + 4];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cq = lane & 15, kg = lane >> 4;
    const int m0 = blockIdx.y * kRows;
    const TileAdapters rows(a, m0, lane);
    const int padded = (a.rank + 31) & ~31;
    for (int row = wave; row < kRows; row += kWaves) {
        const int l = __builtin_amdgcn_readlane(rows.mine, row);
        const float s = l >= 0 ? a.scaling[l] : 0.f;
        for (int r = lane; r < padded; r += 64) {
            float sum = 0.f;
            if (l >= 0 && r < a.rank)
                for (int i = 0; i < a.slices; ++i)
                    sum += a.t[((size_t)i * a.M + m0 + row) * a.rank + r];
            ts[row][r] = s * sum;
        }
    }
    __syncthreads();
    const int n = blockIdx.x * kCols + wave * 16 + cq;
    const int nc = min(n, a.N - 1);
    float4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t left = rows.first; left != 0; left &= left - 1) {
        const int l = __builtin_amdgcn_readlane(rows.mine, __builtin_ctz(left));
        const half_t *lb = a.b + ((size_t)l * a.N + nc) * a.rank;
        float4_t d = {0.f, 0.f, 0.f, 0.f};
        for (int r0 = 0; r0 < a.rank; r0 += 32) {
            const int r = r0 + kg * 8;
            half8_t bv = {};
            if (r < a.rank)
                bv = *reinterpret_cast<const half8_t *>(lb + r);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                d = __builtin_amdgcn_mfma_f32_16x16x4f32(ts[cq][r + j], (float)bv[j], d, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
            acc[r] = __shfl(rows.mine, 4 * kg + r) == l ? d[r] : acc[r];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = 4 * kg + r, m = m0 + row;
        const bool bare = __shfl(rows.mine, row) < 0;
        if (m >= a.M || n >= a.N)
            continue;
        const half_t base = a.base[m * a.ld_base + n];
        a.out[m * a.ld_out + n] = bare ? base : (half_t)((float)base + acc[r]);
    }
}

int row_tiles(int M)
{
    return (M + kRows - 1) / kRows;
}

// Workgroups along the adapters of a tile: a decode step's rows mostly have their own each.
int adapter_slots(int M)
{
    return M <= 64 ? (M < kRows ? M : kRows) : 2;
}

int k_slices(int M, int K)
{
    const int groups = row_tiles(M) * adapter_slots(M);
    int slices = 256 / groups;
    const int most = (K + 511) / 512;
    slices = slices > most ? most : slices;
    return slices < 1 ? 1 : slices;
}

}  // namespace

size_t scratch_bytes(int M, int K, int rank)
{
    return (size_t)k_slices(M, K) * M * rank * sizeof(float);
}

hipError_t launch_lora(const Call &c, void *scratch, hipStream_t stream)
{
    Args a = {};
    a.x = c.x;
    a.a = c.a;
    a.b = c.b;
    a.base = c.base;
    a.scaling = c.scaling;
    a.adapter = c.adapter;
    a.t = static_cast<float *>(scratch);
    a.out = c.out;
    a.ldx = c.ldx;
    a.ld_base = c.ld_base;
    a.ld_out = c.ld_out;
    a.M = c.M;
    a.K = c.K;
    a.N = c.N;
    a.rank = c.rank;
    a.adapters = c.adapters;
    const int steps = (c.K + 31) / 32;
    a.slices = k_slices(c.M, c.K);
    a.slice_steps = (steps + a.slices - 1) / a.slices;
    shrink_kernel<<<dim3(row_tiles(c.M), a.slices, adapter_slots(c.M)), kThreads, 0, stream>>>(a);
    expand_kernel<<<dim3((c.N + kCols - 1) / kCols, row_tiles(c.M)), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace lora
}  // namespace gptq
