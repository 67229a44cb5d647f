// Host side of the products of gemm.h, and the packing of operands whose rows are not 16-byte aligned.
#include "gemm.h"

namespace tig {

// Which tile, and how many ranges of k.  A tile's time per step of 128 bytes of k is taken as proportional to its size, with the
// smaller ones' poorer reuse of operands added (a tile of 128 x 128 as 1.3 quarters, one of 64 x 64 as 2 sixteenths of a
// 256 x 256 one); a launch takes as many rounds as its workgroups need on 256 compute units, and joining ranges costs a
// pass over the partial sums.  The cheapest combination is taken.
GemmPlan gemm_plan(int64_t M, int64_t N, int64_t K, int elem, bool may_split)
{
    const int step = kTileBytes / elem;
    const int64_t steps = (K + step - 1) / step;
    GemmPlan best = {64, 1, (int)(steps > 0 ? steps : 1), 0};
    double best_cost = 1e300;
    const int tiles[3] = {256, 128, 64};
    const double cost_of[3] = {1.0, 0.25 * 1.3, 0.0625 * 2.0};
    const int per_cu[3] = {1, 2, 4};  // workgroups that a compute unit holds at once
    const double unit = elem == 4 ? 4.0 : 0.9;  // us of a 256 x 256 step on one compute unit
    for (int t = 0; t < 3; ++t) {
        const int64_t n_tiles = ((M + tiles[t] - 1) / tiles[t]) * ((N + tiles[t] - 1) / tiles[t]);
        for (int splits = 1; splits <= 64 && splits <= (steps > 0 ? steps : 1); splits *= 2) {
            if (splits > 1 && !may_split)
                break;
            const int64_t per = (steps + splits - 1) / splits;
            // workgroups of one unit share it: a round of `per_cu` on every unit
            const int64_t wgs = n_tiles * splits, full = wgs / (256 * per_cu[t]), rest = wgs % (256 * per_cu[t]);
            const double share = (double)((rest + 255) / 256);
            double cost = (full * per_cu[t] + share) * ((double)per * unit * cost_of[t] + 1.0);
            if (rest > 0 && share < 2.0)  // a workgroup alone on its unit waits for its loads
                cost += (double)per * 0.25;
            if (splits > 1)
                cost += 4.0 + (double)splits * M * N * 8.0 / 4e6;
            if (cost < best_cost) {
                best_cost = cost;
                best = GemmPlan{tiles[t], (int)((steps + per - 1) / (per > 0 ? per : 1)), (int)(per > 0 ? per : 1), 0};
            }
        }
    }
    if (best.splits < 1)
        best.splits = 1;
    best.part_bytes = best.splits > 1 ? (size_t)best.splits * M * gemm_part_ld(N) * 4 : 0;
    return best;
}

namespace {

// A thread takes one 16-byte piece of dst.
template <typename E>
__global__ void __launch_bounds__(256) k_pack(const E *src, int64_t ld_src, E *dst, int64_t ld_dst, int64_t rows, int64_t cols)
{
    constexpr int per = 16 / (int)sizeof(E);
    const int64_t pieces = ld_dst / per, items = rows * pieces;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces, c = i % pieces * per;
        struct alignas(16) Piece {
            E v[per];
        } q;
        const E *p = src + r * ld_src + c;
#pragma unroll
        for (int e = 0; e < per; ++e)
            q.v[e] = c + e < cols ? p[e] : (E)0;
        *(Piece *)(dst + r * ld_dst + c) = q;
    }
}

template <typename E>
__global__ void __launch_bounds__(256) k_zero_rows(E *dst, int64_t ld, int64_t rows, int64_t cols)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (int64_t)gridDim.x * 256)
        dst[i / cols * ld + i % cols] = (E)0;
}

}  // namespace

hipError_t launch_zero_rows(void *dst, int64_t ld, int64_t rows, int64_t cols, int elem, hipStream_t s)
{
    const int64_t blocks = (rows * cols + 255) / 256;
    if (blocks == 0)
        return hipSuccess;
    const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
    if (elem == 4)
        hipLaunchKernelGGL((k_zero_rows<uint32_t>), grid, dim3(256), 0, s, (uint32_t *)dst, ld, rows, cols);
    else
        hipLaunchKernelGGL((k_zero_rows<uint16_t>), grid, dim3(256), 0, s, (uint16_t *)dst, ld, rows, cols);
    return hipGetLastError();
}

hipError_t launch_pack(const void *src, int64_t ld_src, void *dst, int64_t ld_dst, int64_t rows, int64_t cols, int elem, hipStream_t s)
{
    const int64_t items = rows * (ld_dst * elem / 16), blocks = (items + 255) / 256;
    if (items == 0)
        return hipSuccess;
    const dim3 grid((unsigned)(blocks < 16384 ? blocks : 16384));
    if (elem == 4)
        hipLaunchKernelGGL((k_pack<uint32_t>), grid, dim3(256), 0, s, (const uint32_t *)src, ld_src, (uint32_t *)dst, ld_dst, rows, cols);
    else
        hipLaunchKernelGGL((k_pack<uint16_t>), grid, dim3(256), 0, s, (const uint16_t *)src, ld_src, (uint16_t *)dst, ld_dst, rows, cols);
    return hipGetLastError();
}

}  // namespace tig
