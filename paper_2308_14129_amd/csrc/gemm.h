// Products of large matrices on the matrix cores, for the dense layer and the loss over a vocabulary (gfx950):
//
//   C[M x N] = sum over k of A(m, k) B(n, k)
//
// Each operand lies in memory either with k adjacent (kRow: A[m * ld + k]) or with its own index adjacent (kCol: A[k * ld + m]);
// a layer's forward pass is row x row, the gradient of its input row x col, the gradient of its matrix col x col, and no
// operand is transposed in memory.  16-bit types are multiplied 16x16x32, fp32 16x16x4; sums are fp32.
//
// A workgroup takes a tile of BM x BN.  128 bytes of k per row of the tile are staged in LDS at a time, in two buffers that take
// turns: the next 128 bytes are on their way (loads that write LDS themselves) while these are multiplied.
//   kRow: rows of 128 bytes; the 16-byte piece c of row r lies at c ^ (r & 7), so that the sixteen rows that an operand load
//         reads at once lie in different banks.
//   kCol: rows of one k each.  A 16-bit operand is read with the transposing LDS load (16 lanes: four k's of sixteen
//         columns), in pieces of 32 bytes at s ^ (bits of the row) for the same reason; fp32 element by element.
// What lies outside of a matrix reads as zero (offsets outside of the buffer descriptor's extent).  Rows are 16-byte aligned
// and whole 16-byte pieces long: where a caller's are not, the caller packs them first (launch_pack).
//
// Bound by the matrix units and, in short products, by a tile's ends, which nothing runs beside.  8192^3 in bf16: 1302 (row x row),
// 1246 (row x col), 1227 (col x col) TFLOP/s; 8192 x 16384 x 4096 1078, 1130, 1162; fp32 8184 x 38016 x 320 130.
//
// The product is computed as B A^T, so that a lane ends with four adjacent columns of one row of C.
#pragma once

#include <type_traits>

#include "kernels_common.h"

namespace tig {

typedef _Float16 halfx8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef int intx4 __attribute__((ext_vector_type(4)));

enum Form { kRow = 0, kCol = 1 };

constexpr int kTileBytes = 128;  // of k, per step

template <typename T>
struct Mat {
    static constexpr int kPer16 = 16 / sizeof(T);
    static constexpr int kStep = kTileBytes / (int)sizeof(T);  // k's per step
};

__device__ inline void mma16(floatx4 &acc, const intx4 &a, const intx4 &b, __bf16)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
__device__ inline void mma16(floatx4 &acc, const intx4 &a, const intx4 &b, _Float16)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(halfx8, a), __builtin_bit_cast(halfx8, b), acc, 0, 0, 0);
}
__device__ inline void mma16(floatx4 &acc, const intx4 &a, const intx4 &b, float)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(a[j]), __int_as_float(b[j]), acc, 0, 0, 0);
}

// One operand's share of a tile in LDS: BX of its rows, 128 bytes of k.
template <typename T, Form F, int BX, int WAVES>
struct Operand {
    static constexpr int kBytes = BX * kTileBytes;
    static constexpr int kLoads = kBytes / (64 * 16 * WAVES);  // loads of a wavefront per step
    static constexpr int kRowBytes = F == kRow ? kTileBytes : BX * (int)sizeof(T);
    static_assert(kLoads * 64 * 16 * WAVES == kBytes, "");
    static constexpr int kReads = F == kRow ? 1 : (sizeof(T) == 4 ? 4 : 2);  // LDS loads of an operand
    uint32_t off[kLoads];   // byte offset of this lane's piece from the step's base, kBufferNone: outside of the operand's own range
    int at_k[kLoads];       // kRow: byte of k; kCol: k, within the step

    // piece of 32 (64) bytes of row r that lies at place s, and the place of piece s
    static __device__ inline int swizzle(int s, int row)
    {
        if constexpr (sizeof(T) == 4)
            return s ^ ((row >> 2) & 3);
        else if constexpr (BX == 64)
            return s ^ (((row >> 1) & 1) | (((row >> 3) & 1) << 1));
        else
            return s ^ ((row & 3) | (((row >> 3) & 1) << 2));
    }
    static constexpr int kPiece = sizeof(T) == 4 ? 4 : 2;  // 16-byte pieces that move together (kCol)

    // x0: first row of the tile, X: rows of the operand
    __device__ inline void init(int64_t ld, int64_t x0, int64_t X)
    {
        const int lane = lane_id(), wave = wave_id_uniform();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int o = ((wave * kLoads + i) * 64 + lane) * 16, row = o / kRowBytes, at = o % kRowBytes / 16;
            if constexpr (F == kRow) {
                const int c = at ^ (row & 7);
                off[i] = x0 + row < X ? (uint32_t)(row * ld * (int)sizeof(T) + c * 16) : kBufferNone;
                at_k[i] = c * 16;
            } else {
                const int c = swizzle(at / kPiece, row) * kPiece + at % kPiece;
                off[i] = x0 + c * Mat<T>::kPer16 < X ? (uint32_t)(row * ld * (int)sizeof(T) + c * 16) : kBufferNone;
                at_k[i] = row;
            }
        }
    }
    // base: the operand's element (x0, first k of the step); left: k's from there on
    __device__ inline void load(const T *base, int64_t left, char *lds) const
    {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, kBufferAll, kBufferFlags);
        const int wave = wave_id_uniform();
        const int most = left >= Mat<T>::kStep ? 0x7fffffff : (F == kRow ? (int)left * (int)sizeof(T) : (int)left);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t o = at_k[i] < most ? off[i] : kBufferNone;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + (wave * kLoads + i) * 1024), 16, (int)o, 0, 0, 0);
        }
    }
    static __device__ inline int64_t step(int64_t ld) { return F == kRow ? (int64_t)Mat<T>::kStep : (int64_t)Mat<T>::kStep * ld; }

    // the lane's operand of rows x .. x + 15 of the tile, half kk of the step
    static __device__ inline intx4 frag(const char *lds, int x, int kk)
    {
        const int lane = lane_id(), i = lane % 16, g = lane / 16;
        if constexpr (F == kRow) {
            const int row = x + i;
            return *(const intx4 *)(lds + row * kTileBytes + (((kk * 4 + g) ^ (row & 7)) * 16));
        } else if constexpr (sizeof(T) == 4) {
            intx4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = kk * 16 + 4 * g + j;
                v[j] = *(const int *)(lds + row * kRowBytes + swizzle(x / 16, row) * 64 + i * 4);
            }
            return v;
        } else {
            const int row = kk * 32 + 8 * g + i / 4;
            const char *p = lds + row * kRowBytes + swizzle(x / 16, row) * 32 + (i % 4) * 8;
            using LdsPtr = __attribute__((address_space(3))) shortx4 *;
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)p);
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(p + 4 * kRowBytes));  // (rows r and r + 4: the same bits 0, 1, 3)
            intx4 v;
            const auto l = __builtin_bit_cast(__attribute__((ext_vector_type(2))) int, lo);
            const auto h = __builtin_bit_cast(__attribute__((ext_vector_type(2))) int, hi);
            v[0] = l[0], v[1] = l[1], v[2] = h[0], v[3] = h[1];
            return v;
        }
    }
};

template <typename T>
struct GemmArgs {
    const T *A, *B;
    int64_t lda, ldb;
    int64_t M, N, K;
    int tiles_m, tiles_n;
    int splits;       // k is split into this many ranges (blockIdx.y)
    int steps_per;    // steps of a range
    float *part;      // splits > 1: [splits][M][ldp] partial sums
    int64_t ldp;      // (multiple of 4)
};

// A launch's workgroups go round the XCDs: each XCD takes a contiguous share of the tiles, and goes through it in groups of
// eight tile rows, so that what its L2 holds of both operands serves several tiles.
constexpr int kGroupRows = 8;
__device__ inline void tile_of_block(int block, int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int n = tiles_m * tiles_n, xcd = block % 8, q = n / 8, r = n % 8;
    const int t = xcd * q + (xcd < r ? xcd : r) + block / 8;
    const int per = kGroupRows * tiles_n, group = t / per, first = group * kGroupRows;
    const int rows = tiles_m - first < kGroupRows ? tiles_m - first : kGroupRows;
    // (as scalars: a division's result is in a vector register, and descriptors made from it would be one per lane)
    tm = __builtin_amdgcn_readfirstlane(first + t % per % rows);
    tn = __builtin_amdgcn_readfirstlane(t % per / rows);
}

// Where a wavefront's part of a tile lies.
struct TileAt {
    int64_t m0, n0;      // first row and column of the wavefront's part
    int64_t M, N;
    int tm, tn;
    int wm, wn;
};

// What an epilogue does element by element, four adjacent columns of a row at a time, of which `left` exist:
//   row(m), col(n, left)             what it needs of the row, of the columns
//   load(row, n, left)               what it reads at the place
//   store(row, col, read, n, v, left)
// FULL: all four exist.  What the next row reads is on its way while this one is stored.
template <int FM, int FN, class Epi>
__device__ inline void each_four(const TileAt &at, const floatx4 (&acc)[FM][FN], const Epi &epi)
{
    const int lane = lane_id(), i16 = lane % 16, g = lane / 16;
    auto rows = [&](auto full) {
        constexpr bool FULL = decltype(full)::value;
        int left[FN];
        decltype(epi.template col<FULL>(0, 0)) cols[FN];
        decltype(epi.template load<FULL>(epi.row(0), 0, 0)) read[2][FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t n = at.n0 + j * 16 + 4 * g, l = at.N - n;
            left[j] = FULL ? 4 : (l < 4 ? (l > 0 ? (int)l : 0) : 4);
            cols[j] = epi.template col<FULL>(n, left[j]);
        }
        auto fetch = [&](int i) {
            const int64_t m = at.m0 + i * 16 + i16;
            const auto r = epi.row(FULL || m < at.M ? m : at.M - 1);
#pragma unroll
            for (int j = 0; j < FN; ++j)
                read[i & 1][j] = epi.template load<FULL>(r, at.n0 + j * 16 + 4 * g, left[j]);
        };
        fetch(0);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            if (i + 1 < FM)
                fetch(i + 1);
            const int64_t m = at.m0 + i * 16 + i16;
            if (FULL || m < at.M) {
                const auto r = epi.row(m);
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    if (FULL || left[j] > 0)
                        epi.template store<FULL>(r, cols[j], read[i & 1][j], at.n0 + j * 16 + 4 * g, acc[i][j], left[j]);
            }
        }
    };
    if (at.m0 + FM * 16 <= at.M && at.n0 + FN * 16 <= at.N)  // (uniform)
        rows(std::true_type());
    else
        rows(std::false_type());
}
struct Nothing {
};

// This wavefront's loads, into LDS among them, have arrived.
__device__ inline void wait_for_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }  // vmcnt(0)
// A barrier behind which every wavefront's loads into LDS can be read.  (__syncthreads() alone does not promise that: where a
// loop carried the loads over its back edge the compiler waited for them ahead of the loop only.)
__device__ inline void sync_with_loads()
{
    wait_for_loads();
    __syncthreads();
}

struct EpiPart {  // a range's partial sums
    float *part;
    int64_t ldp;
    __device__ inline float *row(int64_t m) const { return part + m * ldp; }
    template <bool FULL>
    __device__ inline Nothing col(int64_t, int) const { return {}; }
    template <bool FULL>
    __device__ inline Nothing load(const float *, int64_t, int) const { return {}; }
    template <bool FULL>
    __device__ inline void store(float *r, Nothing, Nothing, int64_t n, const floatx4 &v, int) const { *(floatx4 *)(r + n) = v; }
};

template <typename T, Form FA, Form FB, int BM, int BN, int WM, int WN, class Epi>
__global__ void __launch_bounds__(64 * WM *WN) k_gemm(GemmArgs<T> g, Epi epi)
{
    constexpr int WAVES = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
    using OA = Operand<T, FA, BM, WAVES>;
    using OB = Operand<T, FB, BN, WAVES>;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int kStage = OA::kBytes + OB::kBytes;
    const int wave = wave_id_uniform(), wm = wave / WN, wn = wave % WN;
    int tm, tn;
    tile_of_block((int)blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int64_t s0 = (int64_t)blockIdx.y * g.steps_per, steps_all = (g.K + Mat<T>::kStep - 1) / Mat<T>::kStep;
    const int64_t s1 = s0 + g.steps_per < steps_all ? s0 + g.steps_per : steps_all;
    OA oa;
    OB ob;
    oa.init(g.lda, m0, g.M);
    ob.init(g.ldb, n0, g.N);
    const T *pa = g.A + (FA == kRow ? m0 * g.lda : m0) + s0 * OA::step(g.lda);
    const T *pb = g.B + (FB == kRow ? n0 * g.ldb : n0) + s0 * OB::step(g.ldb);
    int64_t left = g.K - s0 * Mat<T>::kStep;
    floatx4 acc[FM][FN] = {};
    const int n_steps = (int)(s1 - s0);
    // Two halves of a step take turns: while one's operands are multiplied, the next one's are read from LDS, and between them
    // the step after the next is asked for.  (Read and multiplied in turn, the matrix units waited a third of the time for LDS.)
    intx4 a[2][FM], b[2][FN];
    auto request = [&](int s) {  // (behind the last step: nothing is loaded, and no branch divides the instructions to be mixed)
        char *const to = smem + (s & 1) * kStage;
        oa.load(pa, s < n_steps ? left : 0, to);
        ob.load(pb, s < n_steps ? left : 0, to + OA::kBytes);
        pa += OA::step(g.lda);
        pb += OB::step(g.ldb);
        left -= Mat<T>::kStep;
    };
    constexpr bool kTurned = sizeof(T) == 2 && (FA == kCol || FB == kCol);
    auto multiply = [&](const intx4 (&x)[FM], const intx4 (&y)[FN], intx4 (&nx)[FM], intx4 (&ny)[FN], const char *from, int kk, int s, auto loads) {
        if (decltype(loads)::value && !kTurned)
            request(s);
#pragma unroll
        for (int j = 0; j < FN; ++j)
            ny[j] = OB::frag(from + OA::kBytes, wn * (BN / WN) + j * 16, kk);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            nx[i] = OA::frag(from, wm * (BM / WM) + i * 16, kk);
#pragma unroll
            for (int j = 0; j < FN; ++j)
                mma16(acc[i][j], y[j], x[i], T());
        }
        if (decltype(loads)::value && kTurned)
            request(s);
        // The reads go between the first rows' products: left alone they are sunk to where they are waited for, and ahead of the
        // first product they would be waited for with what it needs.  (Two behind each row's: 3 - 8 % slower.)  So do the next
        // step's loads; the barrier comes as soon as the reads are done, and what is left of the products hides how far
        // the wavefronts are apart (8192^3: with the loads ahead of all products and the barrier behind them 1070, 1030 and 1040
        // instead of 1270, 1145 and 1147 TFLOP/s for the three forms).
        // Transposing reads are another matter: the compiler waits for every load into LDS ahead of them.  So the loads come
        // behind a step's last reads, and the next ones as late as their products allow.
        constexpr int kMma = FN * (sizeof(T) == 4 ? 4 : 1);
        if constexpr (!kTurned) {
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, kMma, 0);
                if (decltype(loads)::value && i < 4)
                    __builtin_amdgcn_sched_group_barrier(0x010, (OA::kLoads + OB::kLoads + 3) / 4, 0);
                if (i + 1 < FM)
                    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
            }
        } else {
            constexpr int kReads = FM * OA::kReads + FN * OB::kReads, kGaps = FM / 2, kFirst = decltype(loads)::value ? 0 : FM / 2 - 1;
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, kMma, 0);
                if (i >= kFirst && i < kFirst + kGaps)
                    __builtin_amdgcn_sched_group_barrier(0x100, (kReads + kGaps - 1) / kGaps, 0);
                if (decltype(loads)::value && i >= kGaps)
                    __builtin_amdgcn_sched_group_barrier(0x010, (OA::kLoads + OB::kLoads + kGaps - 1) / kGaps, 0);
            }
        }
    };
    if (n_steps > 0) {
        request(0);
        sync_with_loads();
        request(1);
#pragma unroll
        for (int i = 0; i < FM; ++i)
            a[0][i] = OA::frag(smem, wm * (BM / WM) + i * 16, 0);
#pragma unroll
        for (int j = 0; j < FN; ++j)
            b[0][j] = OB::frag(smem + OA::kBytes, wn * (BN / WN) + j * 16, 0);
    }
    for (int s = 0; s < n_steps; ++s) {
        multiply(a[0], b[0], a[1], b[1], smem + (s & 1) * kStage, 1, 0, std::false_type());
        sync_with_loads();  // (step s + 1 is there, and nobody reads step s any more)
        multiply(a[1], b[1], a[0], b[0], smem + ((s + 1) & 1) * kStage, 0, s + 2, std::true_type());  // (behind the last step: operands that nobody takes)
    }
    wait_for_loads();  // (nothing may reach LDS any more once the workgroup has given it back)
    const TileAt at = {m0 + wm * (BM / WM), n0 + wn * (BN / WN), g.M, g.N, tm, tn, wm, wn};
    if constexpr (Epi::kWhole) {
        __syncthreads();
        epi.template tile<BM, BN, WM, WN>(at, acc, smem);
    } else if (g.splits > 1) {
        each_four(at, acc, EpiPart{g.part + (int64_t)blockIdx.y * g.M * g.ldp, g.ldp});
    } else {
        each_four(at, acc, epi);
    }
}

// The ranges' partial sums, added in order.
template <class Epi>
__global__ void __launch_bounds__(256) k_gemm_join(const float *part, int splits, int64_t M, int64_t N, int64_t ldp, Epi epi)
{
    const int64_t per = (N + 3) / 4, items = M * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < items; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per, n = i % per * 4;
        floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        const float *p = part + m * ldp + n;
#pragma unroll 8
        for (int s = 0; s < splits; ++s)
            v += *(const floatx4 *)(p + (int64_t)s * M * ldp);
        const int left = N - n < 4 ? (int)(N - n) : 4;
        const auto r = epi.row(m);
        epi.template store<false>(r, epi.template col<false>(n, left), epi.template load<false>(r, n, left), n, v, left);
    }
}

// ---- host side

struct GemmPlan {
    int tile;         // 256, 128 or 64
    int splits, steps_per;
    size_t part_bytes;
};

// which tile, and into how many ranges k is split (see gemm_plan's comment)
GemmPlan gemm_plan(int64_t M, int64_t N, int64_t K, int elem, bool may_split);
inline int64_t gemm_part_ld(int64_t N) { return (N + 3) / 4 * 4; }

// rows of an operand lie as the product reads them (with inner = the adjacent index's extent); offsets inside of a tile, of
// at most 256 rows, stay below 2^31
inline bool gemm_fits(const void *p, int64_t ld, int64_t inner, int elem)
{
    return ((uintptr_t)p & 15) == 0 && ld * elem % 16 == 0 && inner * elem % 16 == 0 && ld * elem <= (1 << 22);
}
constexpr int64_t kMaxDim = 1 << 20;  // of a row that is packed: 4 MiB

template <typename T, Form FA, Form FB, class Epi, int BM, int BN, int WM, int WN>
hipError_t launch_gemm_tile(const GemmPlan &plan, GemmArgs<T> g, const Epi &epi, hipStream_t s)
{
    g.tiles_m = (int)((g.M + BM - 1) / BM);
    g.tiles_n = (int)((g.N + BN - 1) / BN);
    if (g.tiles_m == 0 || g.tiles_n == 0)
        return hipSuccess;
    if ((int64_t)g.tiles_m * g.tiles_n * g.splits * (64 * WM * WN) > 0xffffffff)  // (a launch's threads are counted in 32 bits)
        return hipErrorInvalidValue;
    auto *k = k_gemm<T, FA, FB, BM, BN, WM, WN, Epi>;
    constexpr int lds = 2 * (BM + BN) * kTileBytes;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL(k, dim3((unsigned)(g.tiles_m * g.tiles_n), (unsigned)g.splits), dim3(64 * WM * WN), lds, s, g, epi);
    return hipGetLastError();
}

template <class Epi>
hipError_t launch_join(const float *part, int splits, int64_t M, int64_t N, int64_t ldp, const Epi &epi, hipStream_t s)
{
    const int64_t blocks = (M * ((N + 3) / 4) + 255) / 256;
    hipLaunchKernelGGL((k_gemm_join<Epi>), dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s, part, splits, M, N, ldp, epi);
    return hipGetLastError();
}

// part: plan.part_bytes of device memory (16-byte aligned), if any
template <typename T, Form FA, Form FB, class Epi>
hipError_t launch_gemm(const GemmPlan &plan, const T *A, int64_t lda, const T *B, int64_t ldb, int64_t M, int64_t N, int64_t K, void *part,
                       const Epi &epi, hipStream_t s)
{
    GemmArgs<T> g = {};
    g.A = A, g.B = B, g.lda = lda, g.ldb = ldb, g.M = M, g.N = N, g.K = K;
    g.splits = plan.splits, g.steps_per = plan.steps_per;
    g.part = (float *)part, g.ldp = gemm_part_ld(N);
    hipError_t e;
    if (sizeof(T) == 2 && plan.tile == 256) {
        if constexpr (sizeof(T) == 2)
            e = launch_gemm_tile<T, FA, FB, Epi, 256, 256, 2, 4>(plan, g, epi, s);
    } else if (plan.tile == 128) {
        e = launch_gemm_tile<T, FA, FB, Epi, 128, 128, 2, 2>(plan, g, epi, s);
    } else {
        e = launch_gemm_tile<T, FA, FB, Epi, 64, 64, 2, 2>(plan, g, epi, s);
    }
    if constexpr (!Epi::kWhole)
        if (e == hipSuccess && plan.splits > 1)
            e = launch_join((const float *)part, plan.splits, M, N, g.ldp, epi, s);
    return e;
}

// dst[rows x ld_dst] = src, the columns from `cols` to ld_dst zero.  dst is 16-byte aligned and ld_dst whole 16-byte pieces.
hipError_t launch_pack(const void *src, int64_t ld_src, void *dst, int64_t ld_dst, int64_t rows, int64_t cols, int elem, hipStream_t s);
// rows of zeros
hipError_t launch_zero_rows(void *dst, int64_t ld, int64_t rows, int64_t cols, int elem, hipStream_t s);
// out[n] = alpha * scale (if not NULL) * sum over b < blocks of sums[b * lds + n], added in double
template <typename T>
hipError_t launch_join_sums(const float *sums, int64_t lds, int64_t blocks, int64_t N, T *out, const float *scale, float alpha, hipStream_t s);
inline int64_t pack_ld(int64_t cols, int elem) { return (cols * elem + 15) / 16 * 16 / elem; }

// ---- elements

__device__ inline float to_float(float v) { return v; }
__device__ inline float to_float(__bf16 v) { return (float)v; }
__device__ inline float to_float(_Float16 v) { return (float)v; }

// Four elements as one access, wherever they start: global memory takes accesses at any address.  (An element at a time, the gradient of
// 19599 candidates of 1926 bf16 columns was stored in 86 us instead of 32.)
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Four {
    T v[4];
};

// four adjacent elements (of which `left` exist), rounded to nearest even
template <typename T>
__device__ inline void store_four(T *p, const floatx4 &v, int left)
{
    if (left == 4) {
        *(Four<T> *)p = Four<T>{{(T)v[0], (T)v[1], (T)v[2], (T)v[3]}};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left)
                p[e] = (T)v[e];
    }
}
template <typename T>
__device__ inline floatx4 load_four(const T *p, int left)
{
    floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (left == 4) {
        const Four<T> q = *(const Four<T> *)p;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = to_float(q.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left)
                v[e] = to_float(p[e]);
    }
    return v;
}
// 16 bytes of elements
template <typename T>
__device__ inline void load_piece(const T *p, floatx4 (&v)[Mat<T>::kPer16 / 4])
{
    struct alignas(16) Piece {
        T v[Mat<T>::kPer16];
    };
    const Piece q = *(const Piece *)p;
#pragma unroll
    for (int e = 0; e < Mat<T>::kPer16; ++e)
        v[e / 4][e % 4] = to_float(q.v[e]);
}
template <typename T>
__device__ inline void store_piece(T *p, const floatx4 (&v)[Mat<T>::kPer16 / 4])
{
    struct alignas(16) Piece {
        T v[Mat<T>::kPer16];
    } q;
#pragma unroll
    for (int e = 0; e < Mat<T>::kPer16; ++e)
        q.v[e] = (T)v[e / 4][e % 4];
    *(Piece *)p = q;
}
inline bool piece_aligned(const void *p, int64_t ld, int elem) { return ((uintptr_t)p & 15) == 0 && ld * elem % 16 == 0; }

// C = alpha * sum, alpha from the host times *scale (if not NULL)
template <typename T>
struct EpiStore {
    static constexpr bool kWhole = false;
    T *C;
    int64_t ldc;
    const float *scale;
    float alpha;
    struct Row {
        T *p;
        float by;
    };
    __device__ inline Row row(int64_t m) const { return {C + m * ldc, scale ? alpha * *scale : alpha}; }
    template <bool FULL>
    __device__ inline Nothing col(int64_t, int) const { return {}; }
    template <bool FULL>
    __device__ inline Nothing load(const Row &, int64_t, int) const { return {}; }
    template <bool FULL>
    __device__ inline void store(const Row &r, Nothing, Nothing, int64_t n, const floatx4 &v, int left) const
    {
        store_four(r.p + n, v * r.by, FULL ? 4 : left);
    }
};

}  // namespace tig
