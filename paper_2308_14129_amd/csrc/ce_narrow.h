// Softmax cross entropy over a vocabulary where rows are narrow (16-bit types, at most 128 columns): the logits of a tile and
// what becomes of them stay in registers.  Included by softmax_ce.hip.  KB: blocks of 32 columns that a row has.
//
// With 100 columns a logit costs 200 operations of the matrix units, less than writing and reading it: P in memory (see
// softmax_ce.hip) is what bounds wide rows' way there.  Here a wavefront keeps FM x 16 rows of its OWN matrix as matrix operands and
// streams the other matrix through LDS, 64 rows at a time:
//   statistics   own = rows of X, stream = candidates: running maximum and sum of each lane's share of a row, joined at the end
//   dX           own = rows of X, stream = candidates: dX += P W
//   dW           own = candidates, stream = rows of X: dW += P^T X
// The product of a streamed tile and own rows leaves a lane with 4 + 4 streamed rows (of two sixteens) of one own row: as 16-bit
// values these eight are an operand of the second product as they lie, whose other operand (the streamed rows again, now
// summed over) comes from the same LDS tile with the transposing load.  So each gradient forms the logits once more (10 n V d
// operations instead of 8), and P is never in memory.
//
// Bound by the exponentials and the products, of which a wavefront does one after the other and two wavefronts share a SIMD: 4000 x
// 250000 x 100 in bf16 258 us statistics (775 TFLOP/s of 200 operations a logit), 371 dX, 449 dW (1078 and 891 of 400).
//
// P is rounded to 16 bits for the second product: it is at most 1 in magnitude, relative to the largest weight.
//
// BIASED: both matrices are copies with one column more: W's holds the candidate's bias (-infinity in the rows that fill its last
// tile), X's ones, also in rows that do not count or fill the last tile.  The product adds the bias, and no tile's sums start from
// values that have to be read first.  (The ones' column of dW would be the bias' gradient, but of P as it is rounded for the
// product: the row sums of P before that are added by the vector unit, 4000 x 250000 x 100 in bf16 1061 -> 1067 us.)
#pragma once

#include "gemm.h"

namespace tig {

constexpr int kNarrowWaves = 4, kNarrowStream = 64;
template <int KB>
constexpr int kNarrowOwn = KB <= 2 ? 4 : 3;  // sixteens of own rows of a wavefront (registers: two wavefronts on a SIMD)
template <int KB>
constexpr int kNarrowTile = 16 * kNarrowOwn<KB> * kNarrowWaves;

constexpr float kLog2e = 1.4426950408889634f;
// Logits go to powers of two in one instruction, l log2 e - (largest) log2 e, where the largest is at most this far from zero.  The
// last product is rounded: beyond, where a candidate is masked by a large number, the error would reach the power itself (at -1e9 up to
// 64), and its overflow would make a sum of masked candidates infinite.  There the difference is formed first.
// A gradient's powers, l log2 e - (lse log2 e), are the same: of rows whose lse log2 e is beyond kNarrowFar2 they are formed
// as exp(l - top) / sum.
constexpr float kNarrowFar = 256.0f, kNarrowFar2 = 370.0f;
__device__ inline bool narrow_far(float lse2) { return fabsf(lse2) > kNarrowFar2 && lse2 != INFINITY; }  // (infinity: no probabilities)

template <typename T>
struct NarrowArgs {
    const T *own, *stream;
    int64_t ld_own, ld_stream, n_own, n_stream;
    int d, k;                 // columns of a gradient, of the rows as they are read (BIASED: one more)
    int splits;               // ranges of the streamed rows
    int64_t per;              // tiles of a range
    const float *own_add;     // not BIASED: [n_own] added to an own row's logits (a candidate's bias), or NULL
    const float *stream_add;  // not BIASED: [whole tiles] added to a streamed row's logits, -infinity behind the last, or NULL
    const float *lse2;        // rows of X, for the gradients [whole tiles]: lse log2 e - log2 of P's scale; infinity: no probabilities
    const float *top, *per_sum;  // ... and what far rows take: largest logit (infinity), P's scale over the sum (0)
    const int *some_far;         // is there a far row at all?
    const float *w_stream;    // dW, weighted rows: [whole tiles]
    const int32_t *labels;    // labels of the rows of X (-1: ignored): dX [n_own], dW [whole tiles] (-1 behind the last)
    float p_scale;            // P's scale (1, or 2^14)
    float2 *part;             // statistics: [splits][n_own]
    float *grad;              // [splits][n_own][ld_grad] sums
    int64_t ld_grad;
    float *sums;              // dW: [splits][n_own] row sums of P, or NULL
    EpiStore<T> direct;       // dW in one range: the gradient itself (C NULL: `grad`)
};

// 64 streamed rows of KB x 64 bytes in LDS: the 16-byte piece c of row r lies at c ^ (r mod 16, or mod the pieces of a row)
template <typename T, int KB>
struct NarrowStream {
    static constexpr int kRowBytes = KB * 64, kPieces = KB * 4, kMask = (kPieces < 16 ? kPieces : 16) - 1;
    static constexpr int kBytes = kNarrowStream * kRowBytes;
    uint32_t off[KB];
    int row[KB];
    __device__ inline void init(int64_t ld, int k)
    {
#pragma unroll
        for (int i = 0; i < KB; ++i) {
            const int o = ((wave_id_uniform() * KB + i) * 64 + lane_id()) * 16;
            row[i] = o / kRowBytes;
            const int c = (o % kRowBytes / 16) ^ (row[i] & kMask);
            off[i] = c * 8 < k ? (uint32_t)(row[i] * ld * 2 + c * 16) : kBufferNone;
        }
    }
    __device__ inline void load(const T *base, int64_t left, char *lds) const
    {
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, kBufferAll, kBufferFlags);
        const int most = left < kNarrowStream ? (int)left : kNarrowStream;
#pragma unroll
        for (int i = 0; i < KB; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + (wave_id_uniform() * KB + i) * 1024), 16,
                                                     (int)(row[i] < most ? off[i] : kBufferNone), 0, 0, 0);
    }
    // streamed rows x .. x + 15, columns 32 kk ..
    static __device__ inline intx4 frag(const char *lds, int x, int kk)
    {
        const int i16 = lane_id() % 16, g = lane_id() / 16;
        return *(const intx4 *)(lds + (x + i16) * kRowBytes + (((kk * 4 + g) ^ (i16 & kMask)) * 16));
    }
    // columns 16 t .. 16 t + 15 of the rows x + 4 g .. + 3 and x + 16 + 4 g .. + 3, summed over these
    static __device__ inline intx4 frag_t(const char *lds, int x, int t)
    {
        const int i16 = lane_id() % 16, g = lane_id() / 16, r = 4 * g + i16 / 4;
        const char *p = lds + (x + r) * kRowBytes + (((2 * t + (i16 % 4) / 2) ^ (r & kMask)) * 16) + (i16 & 1) * 8;
        using LdsPtr = __attribute__((address_space(3))) shortx4 *;
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)p);
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(p + 16 * kRowBytes));
        typedef int intx2 __attribute__((ext_vector_type(2)));
        const intx2 l = __builtin_bit_cast(intx2, lo), h = __builtin_bit_cast(intx2, hi);
        return intx4{l[0], l[1], h[0], h[1]};
    }
};

// Where whole rounds of ranges go over the XCDs, the workgroups that stream the same range follow each other on one XCD, whose
// L2 then serves all of them.
__device__ inline void narrow_block(int own_tiles, int splits, int &tile, int &split)
{
    const int b = (int)blockIdx.x, at = splits % 8 == 0 ? b / 8 : b;
    split = __builtin_amdgcn_readfirstlane(splits % 8 == 0 ? b % 8 + 8 * (at / own_tiles) : at / own_tiles);
    tile = __builtin_amdgcn_readfirstlane(at % own_tiles);
}
// Ranges of the streamed rows: about four workgroups for every compute unit, ranges of four tiles at least.
inline int narrow_splits(int64_t own_tiles, int64_t n_stream)
{
    const int64_t tiles = (n_stream + kNarrowStream - 1) / kNarrowStream;
    int64_t s = (1024 + own_tiles - 1) / own_tiles;
    s = s < tiles / 4 ? s : tiles / 4;
    s = s >= 8 ? s / 8 * 8 : s;
    return (int)(s > 1 ? s : 1);
}

template <typename T, int KB, int FM>
__device__ inline void load_own(const NarrowArgs<T> &a, int64_t m0, intx4 (&own)[FM][KB])
{
    const int i16 = lane_id() % 16, g = lane_id() / 16;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t m = m0 + i * 16 + i16;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(a.own + m0 * a.ld_own), 0, kBufferAll, kBufferFlags);
#pragma unroll
        for (int kk = 0; kk < KB; ++kk) {
            const int c = kk * 4 + g;
            const uint32_t o = m < a.n_own && c * 8 < a.k ? (uint32_t)((i * 16 + i16) * a.ld_own * 2 + c * 16) : kBufferNone;
            own[i][kk] = __builtin_bit_cast(intx4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)o, 0, 0));
        }
    }
}

// 64 floats that go with a tile
__device__ inline void load_with(const float *p, int64_t at, char *lds)
{
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(p + at), 0, kNarrowStream * 4, kBufferFlags);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)lds, 4, lane_id() * 4, 0, 0, 0);
}

// what the logits of the four candidates from row r of tile t on start from: their bias, -infinity behind the last candidate
template <bool BIASED, typename T>
__device__ inline floatx4 start_of(const NarrowArgs<T> &a, int64_t t, int r, const char *with)
{
    if constexpr (BIASED)
        return floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    if (a.stream_add)  // (uniform; the table holds -infinity there)
        return *(const floatx4 *)(with + r * 4);
    floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t left = a.n_stream - t * kNarrowStream;
    if (left < kNarrowStream)  // (uniform)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = r + e < left ? 0.0f : -INFINITY;
    return v;
}

template <typename T, int KB, bool BIASED>
__global__ void __launch_bounds__(64 * kNarrowWaves, 2) k_narrow_stats(NarrowArgs<T> a)
{
    constexpr int FM = kNarrowOwn<KB>, FN = 4;
    using S = NarrowStream<T, KB>;
    __shared__ __attribute__((aligned(1024))) char smem[2][S::kBytes + 256];
    int tile, split;
    narrow_block((int)((a.n_own + kNarrowTile<KB> - 1) / kNarrowTile<KB>), a.splits, tile, split);
    const int lane = lane_id(), wave = wave_id_uniform(), i16 = lane % 16, g = lane / 16;
    const int64_t m0 = (int64_t)tile * kNarrowTile<KB> + wave * 16 * FM;
    const int64_t t0 = split * a.per, all = (a.n_stream + kNarrowStream - 1) / kNarrowStream, t1 = t0 + a.per < all ? t0 + a.per : all;
    S st;
    st.init(a.ld_stream, a.k);
    auto request = [&](int64_t t, char *lds) {
        st.load(a.stream + t * kNarrowStream * a.ld_stream, a.n_stream - t * kNarrowStream, lds);
        if (!BIASED && a.stream_add && wave == 0)
            load_with(a.stream_add, t * kNarrowStream, lds + S::kBytes);
    };
    intx4 own[FM][KB];
    load_own<T, KB, FM>(a, m0, own);
    float top[FM], sum[FM];  // in powers of two; this lane's share of its rows
#pragma unroll
    for (int i = 0; i < FM; ++i)
        top[i] = -INFINITY, sum[i] = 0.0f;
    if (t0 < t1)
        request(t0, smem[0]);
    for (int64_t t = t0; t < t1; ++t) {
        const char *const now = smem[(t - t0) & 1];
        sync_with_loads();
        if (t + 1 < t1)
            request(t + 1, smem[(t + 1 - t0) & 1]);
        floatx4 acc[FM][FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const floatx4 from = start_of<BIASED>(a, t, 16 * j + 4 * g, now + S::kBytes);
#pragma unroll
            for (int i = 0; i < FM; ++i)
                acc[i][j] = from;
#pragma unroll
            for (int kk = 0; kk < KB; ++kk) {
                const intx4 f = S::frag(now, 16 * j, kk);
#pragma unroll
                for (int i = 0; i < FM; ++i)
                    mma16(acc[i][j], f, own[i][kk], T());
            }
        }
        float m[FM], most = 0.0f;
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            m[i] = top[i];
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    m[i] = fmaxf(m[i], acc[i][j][v]);
            most = fmaxf(most, fabsf(m[i]));
        }
        auto add = [&](auto some_far) {  // (each lane by its own rule: a row's bits do not depend on its neighbours)
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const float from = m[i] * kLog2e, far_from = m[i] == -INFINITY ? 0.0f : m[i];
                const bool far = decltype(some_far)::value && fabsf(m[i]) > kNarrowFar;
                float s = sum[i] * __builtin_amdgcn_exp2f((far ? top[i] - far_from : top[i] - m[i]) * kLog2e);
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        s += __builtin_amdgcn_exp2f(far ? (acc[i][j][v] - far_from) * kLog2e : fmaf(acc[i][j][v], kLog2e, -from));
                sum[i] = s;
                top[i] = m[i];
            }
        };
        if (__ballot(most > kNarrowFar) == 0ull)
            add(std::false_type());
        else
            add(std::true_type());
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int x = 16; x <= 32; x *= 2) {
            const float om = __shfl_xor(top[i], x), os = __shfl_xor(sum[i], x);
            const float m = fmaxf(top[i], om), from = m == -INFINITY ? 0.0f : m;
            sum[i] = sum[i] * expf(top[i] - from) + os * expf(om - from);
            top[i] = m;
        }
        const int64_t m = m0 + i * 16 + i16;
        if (g == 0 && m < a.n_own)
            a.part[(int64_t)split * a.n_own + m] = make_float2(top[i], sum[i]);
    }
}

// CANDS: own rows are candidates (dW), else rows of X (dX).  WEIGHTED: rows of X have weights of their own.
// DT: sixteens of columns of the gradient.
template <typename T, int KB, int DT, bool BIASED, bool CANDS, bool WEIGHTED>
__global__ void __launch_bounds__(64 * kNarrowWaves, 2) k_narrow_grad(NarrowArgs<T> a)
{
    constexpr int FM = kNarrowOwn<KB>;
    using S = NarrowStream<T, KB>;
    constexpr int kWith = 3 * 256;  // floats that go with a streamed tile: what its logits start from, or lse and weights, labels
    __shared__ __attribute__((aligned(1024))) char smem[2][S::kBytes + kWith];
    int tile, split;
    narrow_block((int)((a.n_own + kNarrowTile<KB> - 1) / kNarrowTile<KB>), a.splits, tile, split);
    const int lane = lane_id(), wave = wave_id_uniform(), i16 = lane % 16, g = lane / 16;
    const int64_t m0 = (int64_t)tile * kNarrowTile<KB> + wave * 16 * FM;
    const int64_t t0 = split * a.per, all = (a.n_stream + kNarrowStream - 1) / kNarrowStream, t1 = t0 + a.per < all ? t0 + a.per : all;
    S st;
    st.init(a.ld_stream, a.k);
    auto request = [&](int64_t t, char *lds) {
        st.load(a.stream + t * kNarrowStream * a.ld_stream, a.n_stream - t * kNarrowStream, lds);
        if constexpr (CANDS) {
            if (wave == 0)
                load_with(a.lse2, t * kNarrowStream, lds + S::kBytes);
            if (wave == 1)
                load_with((const float *)a.labels, t * kNarrowStream, lds + S::kBytes + 256);
            if (WEIGHTED && wave == 2)
                load_with(a.w_stream, t * kNarrowStream, lds + S::kBytes + 512);
        } else {
            if (!BIASED && a.stream_add && wave == 0)
                load_with(a.stream_add, t * kNarrowStream, lds + S::kBytes);
        }
    };
    intx4 own[FM][KB];
    load_own<T, KB, FM>(a, m0, own);
    float mine[FM];  // dX: -lse log2 e of the row; dW: bias of the candidate
    float total[FM] = {};
    int mine_label[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t m = m0 + i * 16 + i16, mm = m < a.n_own ? m : 0;
        if constexpr (CANDS) {
            mine[i] = !BIASED && a.own_add ? a.own_add[mm] : 0.0f;
        } else {
            mine[i] = -a.lse2[mm];
            mine_label[i] = m < a.n_own ? a.labels[mm] : -1;
        }
    }
    floatx4 out[FM][DT] = {};
    if (t0 < t1)
        request(t0, smem[0]);
    auto stream = [&](auto some_far) {
        for (int64_t t = t0; t < t1; ++t) {
            const char *const now = smem[(t - t0) & 1];
            sync_with_loads();
            if (t + 1 < t1)
                request(t + 1, smem[(t + 1 - t0) & 1]);
            const int base = (int)(t * kNarrowStream) + 4 * g;
            bool hot = false;  // a label of one of the rows is among the candidates of this wavefront and tile: seldom
            if constexpr (CANDS) {
                const int label = *(const int *)(now + S::kBytes + 256 + lane * 4);
                hot = __ballot((uint32_t)(label - (int)m0) < (uint32_t)(16 * FM)) != 0ull;
            } else {
#pragma unroll
                for (int i = 0; i < FM; ++i)
                    hot |= (uint32_t)(mine_label[i] - (int)(t * kNarrowStream)) < (uint32_t)kNarrowStream;
                hot = __ballot(hot) != 0ull;
            }
#pragma unroll
            for (int x = 0; x < kNarrowStream; x += 32) {
                intx4 P[FM];
                {
                    floatx4 acc[FM][2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        floatx4 from = {0.0f, 0.0f, 0.0f, 0.0f};
                        if constexpr (!CANDS)
                            from = start_of<BIASED>(a, t, x + 16 * j + 4 * g, now + S::kBytes);
#pragma unroll
                        for (int i = 0; i < FM; ++i)
                            acc[i][j] = CANDS ? floatx4{mine[i], mine[i], mine[i], mine[i]} : from;
#pragma unroll
                        for (int kk = 0; kk < KB; ++kk) {
                            const intx4 f = S::frag(now, x + 16 * j, kk);
#pragma unroll
                            for (int i = 0; i < FM; ++i)
                                mma16(acc[i][j], f, own[i][kk], T());
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        floatx4 lse = {0.0f, 0.0f, 0.0f, 0.0f}, w = lse;
                        const char *const with = now + S::kBytes + (x + 16 * j + 4 * g) * 4;
                        if constexpr (CANDS) {
                            lse = *(const floatx4 *)with;
                            if constexpr (WEIGHTED)
                                w = *(const floatx4 *)(with + 512);
                        }
                        if constexpr (!decltype(some_far)::value) {
#pragma unroll
                            for (int i = 0; i < FM; ++i)
#pragma unroll
                                for (int v = 0; v < 4; ++v)
                                    acc[i][j][v] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][v], kLog2e, CANDS ? -lse[v] : mine[i]));
                        } else {  // (each row by its own rule: its bits do not depend on its neighbours)
#pragma unroll
                            for (int i = 0; i < FM; ++i) {
                                const int m = (int)m0 + i * 16 + i16;
#pragma unroll
                                for (int v = 0; v < 4; ++v) {
                                    const uint32_t r = CANDS ? base + x + 16 * j + v : m < a.n_own ? m : 0;
                                    const float lse2 = CANDS ? lse[v] : -mine[i], l = acc[i][j][v];
                                    acc[i][j][v] = narrow_far(lse2) ? __builtin_amdgcn_exp2f((l - a.top[r]) * kLog2e) * a.per_sum[r]
                                                                    : __builtin_amdgcn_exp2f(fmaf(l, kLog2e, -lse2));
                                }
                                __builtin_amdgcn_sched_barrier(0);  // (seldom taken: no registers for several rows at once)
                            }
                        }
                        if constexpr (!CANDS)
                            if (hot)
#pragma unroll
                                for (int v = 0; v < 4; ++v)
#pragma unroll
                                    for (int i = 0; i < FM; ++i)
                                        acc[i][j][v] -= mine_label[i] == base + x + 16 * j + v ? a.p_scale : 0.0f;
                        if constexpr (CANDS) {
                            if (hot) {
                                const intx4 label = *(const intx4 *)(with + 256);
#pragma unroll
                                for (int v = 0; v < 4; ++v)
#pragma unroll
                                    for (int i = 0; i < FM; ++i)
                                        acc[i][j][v] -= label[v] == (int)(m0 + i * 16 + i16) ? a.p_scale : 0.0f;
                            }
#pragma unroll
                            for (int i = 0; i < FM; ++i) {
                                if constexpr (WEIGHTED)
                                    acc[i][j] *= w;
                                if (a.sums)
                                    total[i] += (acc[i][j][0] + acc[i][j][1]) + (acc[i][j][2] + acc[i][j][3]);
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < FM; ++i) {
                        typedef T eight __attribute__((ext_vector_type(8)));
                        eight q;
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            q[v] = (T)acc[i][0][v], q[4 + v] = (T)acc[i][1][v];
                        P[i] = __builtin_bit_cast(intx4, q);
                    }
                }
#pragma unroll
                for (int c = 0; c < DT; ++c) {
                    const intx4 f = S::frag_t(now, x, c);
#pragma unroll
                    for (int i = 0; i < FM; ++i)
                        mma16(out[i][c], f, P[i], T());
                }
            }
        }
    };
    // (two loops: the far rows' instructions in the usual one cost it its registers, 581 -> 717 us at 1000 x 400000 x 128 in bf16)
    if (__builtin_amdgcn_readfirstlane(*a.some_far) == 0)
        stream(std::false_type());
    else
        stream(std::true_type());
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t m = m0 + i * 16 + i16;
        if (CANDS && a.sums) {
            total[i] += __shfl_xor(total[i], 16);
            total[i] += __shfl_xor(total[i], 32);
            if (g == 0 && m < a.n_own)
                a.sums[(int64_t)split * a.n_own + m] = total[i];
        }
        if (m < a.n_own && CANDS && a.direct.C) {
            const auto by = a.direct.row(m);
#pragma unroll
            for (int c = 0; c < DT; ++c)
                if (c * 16 + 4 * g < a.d)
                    a.direct.template store<false>(by, Nothing(), Nothing(), c * 16 + 4 * g, out[i][c], a.d - c * 16 - 4 * g < 4 ? a.d - c * 16 - 4 * g : 4);
        } else if (m < a.n_own && a.grad) {
            float *const row = a.grad + ((int64_t)split * a.n_own + m) * a.ld_grad;
#pragma unroll
            for (int c = 0; c < DT; ++c)
                if (c * 16 + 4 * g < a.d)
                    *(floatx4 *)(row + c * 16 + 4 * g) = out[i][c];
        }
    }
}

}  // namespace tig
