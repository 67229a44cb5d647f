// Host side of the products of gemm.h, and the packing of operands whose rows are not 16-byte aligned.
#include "gemm.h"

#include <cmath>

namespace tig {

// Which tile, and how many ranges of k: the cheapest by this estimate, in us.  A compute unit holds four workgroups of tiles of 64,
// two of 128, one of 256; a round of them takes, per step of 128 bytes of k, `loaded` for each workgroup on the unit and never
// less than `alone`, and `fixed` + `each` for every workgroup at its ends.  No launch is faster than its operands' way from the caches
// at 14 TB/s, and joining ranges costs a launch and 8 bytes per element and range at 6.8 TB/s.  The constants are a fit to 690
// timings (27 products in 16 bits, 15 in fp32, of 8 to 470,816 rows, each in every tile and 1 to 256 ranges): the tile and ranges that it
// takes are within 0.5 % (16 bits) and 1.5 % (fp32) of the fastest on average.  Examples: 669 x 512 x 17024 in fp16 takes 36 us as
// 128 x 128 x 16 ranges, 43 as 256 x 16, 50 as 64 x 4, 74 as 128 x 4; 8192 x 8192 x 2048 in bf16 224 as 256, 310 as 128, 415 as 64;
// 4096 x 320 x 8184 in fp32 174 as 64 x 4, 260 as 256 x 8.  In fp32 a tile of 256 was never the fastest and is not built.
GemmPlan gemm_plan(int64_t M, int64_t N, int64_t K, int elem, bool may_split)
{
    struct Tile {
        int size, per_cu;
        double loaded, alone, fixed, each;
    };
    static const Tile tiles16[3] = {{256, 1, 1.6, 1.6, 6.5, 1.9}, {128, 2, 0.55, 1.1, 4.1, 0.9}, {64, 4, 0.29, 0.37, 3.2, 0.2}};
    static const Tile tiles32[2] = {{128, 2, 1.6, 3.2, 4.1, 0.9}, {64, 4, 0.5, 0.6, 3.2, 0.2}};
    const Tile *const tiles = elem == 4 ? tiles32 : tiles16;
    const int step = kTileBytes / elem;
    const int64_t steps = K > 0 ? (K + step - 1) / step : 1;
    GemmPlan best = {64, 1, (int)steps, 0};
    double best_cost = 1e300;
    for (int i = 0; i < (elem == 4 ? 2 : 3); ++i) {
        const Tile &t = tiles[i];
        const int64_t n_tiles = ((M + t.size - 1) / t.size) * ((N + t.size - 1) / t.size);
        for (int splits = 1; splits <= (may_split ? 256 : 1) && splits <= steps; splits *= 2) {
            const int64_t per = (steps + splits - 1) / splits, ranges = (steps + per - 1) / per;
            const int64_t wgs = n_tiles * ranges, full = wgs / (256 * t.per_cu), share = (wgs % (256 * t.per_cu) + 255) / 256;
            auto round = [&](int64_t n) { return n > 0 ? (double)per * fmax(t.alone, (double)n * t.loaded) + t.fixed + (double)n * t.each : 0.0; };
            double cost = fmax((double)full * round(t.per_cu) + round(share), (double)wgs * per * 2 * t.size * kTileBytes / 14e6);
            if (ranges > 1)
                cost += 3.0 + (double)ranges * M * N * 8.0 / 6.8e6;
            if (cost < best_cost) {
                best_cost = cost;
                best = GemmPlan{t.size, (int)ranges, (int)per, 0};
            }
        }
    }
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
        struct __attribute__((packed, aligned(sizeof(E)))) Piece {  // (read wherever it starts)
            E v[per];
        } q;
        const E *p = src + r * ld_src + c;
        if (c + per <= cols)
            q = *(const Piece *)p;
        else
#pragma unroll
            for (int e = 0; e < per; ++e)
                q.v[e] = c + e < cols ? p[e] : (E)0;
        *(Piece *)__builtin_assume_aligned(dst + r * ld_dst + c, 16) = q;
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
