// Softmax cross entropy of rows over a vocabulary of candidates, with its gradient (include/tig.h, tig_softmax_ce_*).  gfx950.
//
//   statistics   a tile product X W^T (gemm.h) whose epilogue leaves, for every row and tile of candidates, the largest logit and
//                the sum of exp(l - largest); k_ce_rows joins them to the row's log-sum-exp and takes the label's logit
//   gradient     for one piece of the vocabulary after the other: the logits once more, P = w_i (softmax - [label]) in their
//                epilogue, and two tile products, dX += P W and dW = P^T X.  A piece of P stays within the last-level cache.
// s_i = S w_i with S the largest |s_i|: P holds values of at most 1, the products are scaled by S afterwards.
// 8192 x 128000 x 2048 in bf16: statistics 3.51 ms (1.23 PFLOP/s), P 4.04 (1.06), dX 3.71 (1.16), dW 3.81 (1.13).  P is a matrix operand
// and so of the matrices' type: at most 1 in magnitude, relative to the largest weight; fp16 scaled by 2^14 (kPScale).
// Many rows of at most 128 columns in 16-bit types go the way of ce_narrow.h (ce_plan).
#include "act.h"
#include "ce_narrow.h"
#include "gemm.h"

namespace tig {

namespace {

struct CeHead {
    float S;       // largest |s_i|
    int some_far;  // narrow rows: is one of them far (ce_narrow.h)?
};
// What the epilogue of P needs of a row: the largest logit (+infinity: no probabilities), w_i * P's scale over the sum of exponentials and
// by itself, the label (-1: ignored).  (Not the log-sum-exp: where a row's logits are far from zero its rounding would go into
// every probability; all candidates masked by -1e9 had 1 each instead of 1 / V.)
struct alignas(16) CeRow {
    float top, per_sum, w;
    int32_t label;
};

template <typename T>
constexpr float kPScale = 1.0f;
template <>
constexpr float kPScale<_Float16> = 16384.0f;  // (2^14: P's smallest fp16 values stand for 4e-9 in full precision)

template <typename T>
__device__ inline float exp_of(float x)
{
    if constexpr (sizeof(T) == 4)
        return expf(x);
    else
        return __expf(x);
}

// the largest |s_i| where rows have weights of their own
__global__ void __launch_bounds__(1024) k_ce_top(const int32_t *labels, const float *row_scale, float scale, int64_t rows, int64_t vocab, CeHead *head)
{
    __shared__ float top_of[16];
    float top = 0.0f;
    for (int64_t i = threadIdx.x; i < rows; i += 1024)
        if (labels[i] >= 0 && labels[i] < vocab)
            top = fmaxf(top, fabsf(row_scale[i]));
    for (int d = 32; d > 0; d >>= 1)
        top = fmaxf(top, __shfl_xor(top, d));
    if (lane_id() == 0)
        top_of[wave_id()] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w)
            top = fmaxf(top, top_of[w]);
        head->S = top * fabsf(scale);
    }
}

// number of rows that count; their mean loss, in double, always in the same order; S without weights; lse2: narrow rows', or NULL
__global__ void __launch_bounds__(1024) k_ce_mean(const float *loss, const int32_t *labels, int64_t rows, int64_t vocab, bool weighted, float scale,
                                                  const float *lse2, CeHead *head, float *mean)
{
    __shared__ double part[1024];
    __shared__ int count[1024];
    __shared__ bool some_far[16];
    double total = 0.0;
    int n = 0;
    bool far = false;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        total += (double)loss[i];
        n += labels[i] >= 0 && labels[i] < vocab;
        far |= lse2 && narrow_far(lse2[i]);
    }
    part[threadIdx.x] = total;
    count[threadIdx.x] = n;
    far = __ballot(far) != 0ull;
    if (lane_id() == 0)
        some_far[wave_id()] = far;
    __syncthreads();
    for (int d = 512; d > 0; d >>= 1) {
        if ((int)threadIdx.x < d) {
            part[threadIdx.x] += part[threadIdx.x + d];
            count[threadIdx.x] += count[threadIdx.x + d];
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        n = count[0] > 0 ? count[0] : 1;
        if (mean)
            *mean = (float)(part[0] / (double)n);
        if (!weighted)
            head->S = fabsf(scale) / (float)n;
        for (int w = 1; lse2 && w < 16; ++w)
            far |= some_far[w];
        head->some_far = far;
    }
}

// Largest logit and sum of exponentials of a row over a tile of candidates: over a lane's columns, the four lanes of a row, and
// the wavefronts side by side (in LDS).  part[tile][row].
template <typename T>
struct EpiStats {
    static constexpr bool kWhole = true;
    const T *bias;
    float2 *part;
    int64_t rows;
    template <int BM, int BN, int WM, int WN, int FM, int FN>
    __device__ inline void tile(const TileAt &at, floatx4 (&acc)[FM][FN], char *smem) const
    {
        float2 *const red = (float2 *)smem;  // [WN][BM]
        const int lane = lane_id(), i16 = lane % 16, g = lane / 16;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t n = at.n0 + j * 16 + 4 * g;
            const int left = at.N - n < 4 ? (at.N > n ? (int)(at.N - n) : 0) : 4;
            floatx4 b = {0.0f, 0.0f, 0.0f, 0.0f};
            if (bias)
                b = load_four(bias + n, left);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < FM; ++i)
                    acc[i][j][e] = e < left ? acc[i][j][e] + b[e] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    top = fmaxf(top, acc[i][j][e]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float from = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    sum += exp_of<T>(acc[i][j][e] - from);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (g == 0)
                red[at.wn * BM + at.wm * (BM / WM) + i * 16 + i16] = make_float2(top, sum);
        }
        __syncthreads();
        for (int r = threadIdx.x; r < BM; r += 64 * WM * WN) {
            float2 v = red[r];
#pragma unroll
            for (int w = 1; w < WN; ++w) {
                const float2 o = red[w * BM + r];
                const float top = fmaxf(v.x, o.x), from = top == -INFINITY ? 0.0f : top;
                v = make_float2(top, v.y * expf(v.x - from) + o.y * expf(o.x - from));
            }
            const int64_t m = (int64_t)at.tm * BM + r;
            if (m < rows)
                part[(int64_t)at.tn * rows + m] = v;
        }
    }
};

// LANES threads a row: the tiles' parts joined, the label's logit, loss; for the gradient the row's
// record, or the tables that ce_narrow.h streams (whole tiles: rows behind the last take no part), and the row itself where it
// counts, else zeros: whatever it holds, P^T X does not see it.
template <typename T>
struct CeRowsOut {
    float *loss, *lse;
    CeRow *rec;
    float *lse2, *top, *per_sum, *w;  // narrow
    int32_t *label;
    T *x0;
    int64_t ld_x0;
    bool ones;         // a column of ones behind x0's last, also in rows that do not count and behind the last
};
template <typename T, int LANES>
__global__ void __launch_bounds__(256) k_ce_rows(const float2 *part, int64_t tiles, int64_t rows, const T *x, int64_t ldx, const T *w, int64_t ldw,
                                                 const T *bias, int64_t dim, int64_t vocab, const int32_t *labels, const float *row_scale, float scale,
                                                 const CeHead *head, CeRowsOut<T> out)
{
    const int64_t i = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int t = threadIdx.x % LANES;
    const bool on = i < rows;
    const int64_t r = on ? i : rows - 1;
    float top = -INFINITY, sum = 0.0f;
    for (int64_t k = t; k < tiles; k += 4 * LANES) {
        float2 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t at = k + u * LANES;
            v[u] = part[(at < tiles ? at : t) * rows + r];
            if (at >= tiles)
                v[u] = float2{-INFINITY, 0.0f};
        }
        const float to = fmaxf(fmaxf(fmaxf(top, v[0].x), v[1].x), fmaxf(v[2].x, v[3].x)), from = to == -INFINITY ? 0.0f : to;
        sum *= expf(top - from);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            sum += v[u].y * expf(v[u].x - from);
        top = to;
    }
    const int32_t label = labels[r];
    const bool counts = label >= 0 && label < vocab;
    float dot = 0.0f;
    const T *xr = x + r * ldx, *wr = w + (counts ? (int64_t)label : 0) * ldw;
#pragma unroll 4
    for (int64_t k = t; k < dim; k += LANES)
        dot += to_float(xr[k]) * to_float(wr[k]);
    for (int d = LANES / 2; d > 0; d >>= 1) {
        const float ot = __shfl_xor(top, d), os = __shfl_xor(sum, d);
        const float to = fmaxf(top, ot), from = to == -INFINITY ? 0.0f : to;
        sum = sum * expf(top - from) + os * expf(ot - from);
        top = to;
        dot += __shfl_xor(dot, d);
    }
    if (out.x0 && (on || out.ones))  // (rows of x are whole 16-byte pieces here)
        for (int64_t c = t * Mat<T>::kPer16; c < out.ld_x0; c += LANES * Mat<T>::kPer16) {
            union {
                intx4 q;
                T v[Mat<T>::kPer16];
            } u;
            u.q = on && counts && c < dim ? *(const intx4 *)(xr + c) : intx4{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < Mat<T>::kPer16; ++e)
                u.v[e] = out.ones && c + e == dim ? (T)1.0f : u.v[e];
            *(intx4 *)(out.x0 + i * out.ld_x0 + c) = u.q;
        }
    if (t != 0)
        return;
    const float lse = top == -INFINITY && sum == 0.0f ? -INFINITY : top + logf(sum);
    if (on) {
        if (bias && counts)
            dot += to_float(bias[label]);
        if (out.lse)
            out.lse[i] = lse;
        if (out.loss)
            out.loss[i] = !counts ? 0.0f : (dot == -INFINITY ? INFINITY : (top - dot) + logf(sum));  // (far from zero, lse has lost what the sum says)
    }
    if (!out.rec && !out.lse2)
        return;
    float wi = 0.0f;
    if (on && counts)
        wi = row_scale ? (head->S > 0.0f ? row_scale[i] * scale / head->S : 0.0f) : (scale < 0.0f ? -1.0f : 1.0f);
    const bool none = wi == 0.0f || lse == -INFINITY;
    if (out.rec) {
        if (on)
            out.rec[i] = CeRow{none ? INFINITY : top, none ? 0.0f : wi * kPScale<T> / sum, wi * kPScale<T>, wi != 0.0f ? label : -1};
    } else {
        constexpr float shift = sizeof(T) == 2 && kPScale<T> != 1.0f ? 14.0f : 0.0f;
        out.lse2[i] = none ? INFINITY : fmaf(top, kLog2e, log2f(sum)) - shift;
        out.top[i] = none ? INFINITY : top;
        out.per_sum[i] = none ? 0.0f : kPScale<T> / sum;
        out.w[i] = wi;
        out.label[i] = wi != 0.0f ? label : -1;
    }
}

// P of a piece of the vocabulary from v0 on, columns up to a whole 16-byte piece zero; sums: the column sums of P over the tile's
// rows, before rounding (over a lane's rows, the sixteen lanes of a column, and the wavefronts on top of each other).
template <typename T>
struct EpiP {
    static constexpr bool kWhole = true;
    const T *bias;
    const CeRow *rec;
    T *P;
    int64_t ldp, v0;
    float *sums;  // [tiles_m][ldp] or NULL
    template <int BM, int BN, int WM, int WN, int FM, int FN>
    __device__ inline void tile(const TileAt &at, floatx4 (&acc)[FM][FN], char *smem) const
    {
        const int lane = lane_id(), i16 = lane % 16, g = lane / 16;
        const int64_t end = (at.N + Mat<T>::kPer16 - 1) / Mat<T>::kPer16 * Mat<T>::kPer16;
        floatx4 b[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int64_t n = at.n0 + j * 16 + 4 * g;
            const int left = at.N - n < 4 ? (at.N > n ? (int)(at.N - n) : 0) : 4;
            b[j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            if (bias)
                b[j] = load_four(bias + n, left);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                b[j][e] = e < left ? b[j][e] : -INFINITY;
        }
        // the rows' records, by way of LDS: behind a store to P each would wait for memory by itself
        CeRow *const of_row = (CeRow *)(smem + WM * BN * sizeof(float));
        for (int r = threadIdx.x; r < BM; r += 64 * WM * WN) {
            const int64_t m = (int64_t)at.tm * BM + r;
            of_row[r] = m < at.M ? rec[m] : CeRow{INFINITY, 0.0f, 0.0f, -1};
        }
        __syncthreads();
        floatx4 total[FN] = {};
        auto rows = [&](auto full) {
            constexpr bool FULL = decltype(full)::value;
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int64_t m = at.m0 + i * 16 + i16;
                const bool on = FULL || m < at.M;
                const CeRow r = of_row[at.wm * (BM / WM) + i * 16 + i16];
                T *const row = P + m * ldp + at.n0 + 4 * g;
                const int64_t from = (int64_t)r.label - v0 - at.n0 - 4 * g;
                const int hot = r.label >= 0 && from >= 0 && from < 16 * FN ? (int)from : -1;  // (of this lane's columns 16 j + e)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    floatx4 p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[e] = r.top != INFINITY ? exp_of<T>(acc[i][j][e] + b[j][e] - r.top) : 0.0f;
                        p[e] = fmaf(p[e], r.per_sum, hot == 16 * j + e ? -r.w : 0.0f);
                    }
                    total[j] += p;
                    if (FULL || (on && at.n0 + j * 16 + 4 * g < end))
                        store_four(row + j * 16, p, 4);
                }
                __builtin_amdgcn_sched_barrier(0);  // (a row after the other: their values at once do not fit the registers)
            }
        };
        if (at.m0 + FM * 16 <= at.M && at.n0 + FN * 16 <= at.N)  // (uniform)
            rows(std::true_type());
        else
            rows(std::false_type());
        if (!sums)
            return;
        float *const red = (float *)smem;  // [WM][BN]
#pragma unroll
        for (int j = 0; j < FN; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                total[j][e] = row_sum_all(total[j][e]);
            if (i16 == 0)
                *(floatx4 *)(red + at.wm * BN + at.wn * (BN / WN) + j * 16 + 4 * g) = total[j];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < BN; c += 64 * WM * WN) {
            float total = red[c];
#pragma unroll
            for (int w = 1; w < WM; ++w)
                total += red[w * BN + c];
            const int64_t n = (int64_t)at.tn * BN + c;
            if (n < at.N)
                sums[(int64_t)at.tm * ldp + n] = total;
        }
    }
};

// a piece's share of dX: stored, or added to the pieces before it
struct EpiAdd {
    static constexpr bool kWhole = false;
    float *acc;
    int64_t ld;
    bool first;
    __device__ inline float *row(int64_t m) const { return acc + m * ld; }
    template <bool FULL>
    __device__ inline Nothing col(int64_t, int) const { return {}; }
    template <bool FULL>
    __device__ inline floatx4 load(const float *r, int64_t n, int left) const
    {
        return first || left == 0 ? floatx4{0.0f, 0.0f, 0.0f, 0.0f} : *(const floatx4 *)(r + n);
    }
    template <bool FULL>
    __device__ inline void store(float *r, Nothing, const floatx4 &before, int64_t n, const floatx4 &v, int) const { *(floatx4 *)(r + n) = before + v; }
};

template <typename T>
__global__ void __launch_bounds__(256) k_ce_dx(const float *acc, int64_t ld, int64_t rows, int64_t dim, const float *scale, float alpha, T *dx,
                                               int64_t lddx)
{
    const int64_t per = (dim + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per, n = i % per * 4;
        const floatx4 v = *(const floatx4 *)(acc + m * ld + n) * (alpha * *scale);
        store_four(dx + m * lddx + n, v, dim - n < 4 ? (int)(dim - n) : 4);
    }
}

// narrow rows: dX = S w_i (sum of P W over all ranges)
template <typename T>
__global__ void __launch_bounds__(256) k_ce_narrow_dx(const float *grad, int splits, int64_t ld, int64_t rows, int64_t dim, const float *weight,
                                                      const CeHead *head, float alpha, T *dx, int64_t lddx)
{
    const int64_t per = (dim + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per, n = i % per * 4;
        floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
        for (int s = 0; s < splits; ++s)
            v += *(const floatx4 *)(grad + ((int64_t)s * rows + m) * ld + n);
        store_four(dx + m * lddx + n, v * (alpha * head->S * weight[m]), dim - n < 4 ? (int)(dim - n) : 4);
    }
}

// A copy with a column more (`extra`, or `fill` where that is NULL) and rows up to whole tiles: zeros and, in that column, `behind`.
// A thread takes one 16-byte piece.
template <typename T>
__global__ void __launch_bounds__(256) k_ce_copy(const T *src, int64_t ld_src, int64_t rows, int64_t cols, const T *extra, float fill, float behind, T *dst,
                                                 int64_t ld_dst, int64_t all)
{
    constexpr int per = Mat<T>::kPer16;
    const int64_t pieces = ld_dst / per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / pieces, c = i % pieces * per;
        struct __attribute__((packed, aligned(sizeof(T)))) Piece {  // (read wherever it starts)
            T v[per];
        } q;
        const T *p = src + r * ld_src + c;
        if (c + per <= cols && r < rows)
            q = *(const Piece *)p;
        else
#pragma unroll
            for (int e = 0; e < per; ++e)
                q.v[e] = c + e < cols && r < rows ? p[e] : c + e != cols ? (T)0.0f : r >= rows ? (T)behind : extra ? extra[r] : (T)fill;
        *(Piece *)__builtin_assume_aligned(dst + r * ld_dst + c, 16) = q;
    }
}

// a bias in fp32, -infinity behind its last (whole tiles)
template <typename T>
__global__ void __launch_bounds__(256) k_ce_bias(const T *bias, int64_t vocab, float *out, int64_t all)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < all)
        out[i] = i < vocab ? to_float(bias[i]) : -INFINITY;
}

inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct CePlan {
    bool grad, pack_x, pack_w;
    int64_t ld_x, ld_w;      // of the packed copies
    int64_t stat_rows;       // rows whose statistics are formed at a time
    GemmPlan stat;
    int64_t piece;           // candidates of a piece
    GemmPlan logits, dx, dw;
    int64_t ldp, ld_acc;
    bool acc;                // more than one piece: dX in fp32 first
    // narrow rows
    int kb;                  // 32-column blocks of a row (0: not narrow)
    bool biased;             // copies with a column more (ce_narrow.h)
    int64_t own_rows, own_cands;  // tiles of own rows
    int s_stat, s_dx, s_dw;  // ranges of the streamed rows
    int64_t row_tiles, cand_tiles;  // whole tiles of 64
    size_t bias32, lse2, top, per_sum, weight;
    size_t head, loss, rec, label, part, px, pw, px0, P, dxa, join, sums;
    size_t bytes;
};

constexpr size_t kStatBytes = (size_t)256 << 20;   // of parts at a time
constexpr size_t kPieceBytes = (size_t)128 << 20;  // of P at a time: half of the last-level cache

CePlan ce_plan(const tig_softmax_ce &p)
{
    CePlan L = {};
    const int es = dtype_bytes(p.dtype);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += align_up(bytes);
        return at;
    };
    const int64_t n = p.rows, V = p.vocab, d = p.dim;
    L.grad = p.dx || p.dw || p.dbias;
    L.head = take(sizeof(CeHead));
    L.loss = take(4 * (size_t)n);
    L.ld_x = L.ld_w = pack_ld(d, es);
    if (n == 0) {
        L.bytes = off;
        return L;
    }
    // Narrow rows stay in registers where there are enough logits for that to count (us, with gradients, this way and by tiles: 1024 x
    // 30000 x 128 128 and 107, x 100 111 and 119; 128 x 262144 x 128 175 and 178, x 64 142 and 141; 128 x 400000 x 128 217 and 262;
    // 256 x 400000 x 64 193 and 325; 4000 x 250000 x 100 1070 and 3007), and without a gradient over many candidates (8 x 400000 x 64
    // 39 and 47; 512 x 30000 x 64 19 and 17).
    if (es == 2 && d <= 128 && (n * V >= (int64_t)1 << 25 || (!L.grad && V >= 1 << 17))) {
        L.kb = d <= 64 ? 2 : 4;  // (a column more does not change it)
        const int64_t tile = L.kb == 2 ? kNarrowTile<2> : kNarrowTile<4>;
        L.own_rows = (n + tile - 1) / tile, L.own_cands = (V + tile - 1) / tile;
        L.row_tiles = (n + kNarrowStream - 1) / kNarrowStream, L.cand_tiles = (V + kNarrowStream - 1) / kNarrowStream;
        // A column more, where the blocks have room for one and W is copied anyway, or where rows are many (with and without, aligned
        // rows: 300 x 250000 x 120 205 and 188 us, 1024 x 250000 x 96 344 and 335, 1500 x 100000 x 120 265 and 264, 1500 x 250000 x 40
        // 329 and 332, 2000 x 250000 x 96 581 and 582, x 40 405 and 410, 8000 x 100000 x 120 962 and 985).
        const bool fits = gemm_fits(p.w, p.ldw, d, es);
        L.biased = d < 32 * L.kb && (!fits || n >= 2000);
        L.pack_x = L.biased || !gemm_fits(p.x, p.ldx, d, es);
        L.pack_w = L.biased || !fits;
        L.ld_x = L.ld_w = pack_ld(L.biased ? d + 1 : d, es);
        if (L.pack_x)
            L.px = take((size_t)n * L.ld_x * es);
        if (L.pack_w)
            L.pw = take((size_t)L.cand_tiles * kNarrowStream * L.ld_w * es);
        L.s_stat = L.s_dx = narrow_splits(L.own_rows, V);
        L.s_dw = narrow_splits(L.own_cands, n);
        L.stat_rows = n;
        L.part = take((size_t)L.s_stat * n * sizeof(float2));
        if (p.bias && !L.biased)
            L.bias32 = take((size_t)L.cand_tiles * kNarrowStream * 4);
        if (L.grad) {
            const size_t tab = (size_t)L.row_tiles * kNarrowStream * 4;
            L.lse2 = take(tab);
            L.top = take(tab);
            L.per_sum = take(tab);
            L.weight = take(tab);
            L.label = take(tab);
            L.px0 = take((size_t)L.row_tiles * kNarrowStream * L.ld_x * es);
            L.ld_acc = (d + 3) / 4 * 4;
            if (p.dx)
                L.dxa = take((size_t)L.s_dx * n * L.ld_acc * 4);
            if (p.dw && L.s_dw > 1)
                L.join = take((size_t)L.s_dw * V * L.ld_acc * 4);
            if (p.dbias)
                L.sums = take((size_t)L.s_dw * V * 4);
        }
        L.bytes = off;
        return L;
    }
    L.pack_x = !gemm_fits(p.x, p.ldx, d, es);
    L.pack_w = !gemm_fits(p.w, p.ldw, d, es);
    if (L.pack_x)
        L.px = take((size_t)n * L.ld_x * es);
    if (L.pack_w)
        L.pw = take((size_t)V * L.ld_w * es);
    L.stat = gemm_plan(n, V, d, es, false);
    const int64_t tiles = (V + L.stat.tile - 1) / L.stat.tile;
    int64_t most = (int64_t)(kStatBytes / 8) / tiles / 256 * 256;
    if (most < 256)
        most = 256;
    L.stat_rows = n < most ? n : most;
    L.part = take((size_t)L.stat_rows * tiles * sizeof(float2));
    if (L.grad) {
        L.rec = take(sizeof(CeRow) * (size_t)n);
        int64_t piece = (int64_t)(kPieceBytes / es) / n / 256 * 256;
        if (piece < 256)
            piece = 256;
        L.piece = V < piece ? V : piece;
        L.ldp = pack_ld(L.piece, es);
        L.P = take((size_t)n * L.ldp * es);
        L.acc = L.piece < V;
        L.logits = gemm_plan(n, L.piece, d, es, false);
        L.dx = gemm_plan(n, d, L.piece, es, true);
        L.dw = gemm_plan(L.piece, d, n, es, true);
        L.ld_acc = (d + 3) / 4 * 4;
        if (p.dx && L.acc)
            L.dxa = take((size_t)n * L.ld_acc * 4);
        if (p.dw)
            L.px0 = take((size_t)n * L.ld_x * es);
        size_t join = p.dx ? L.dx.part_bytes : 0;
        if (p.dw && L.dw.part_bytes > join)
            join = L.dw.part_bytes;
        L.join = take(join);
        if (p.dbias)
            L.sums = take((size_t)((n + L.logits.tile - 1) / L.logits.tile) * L.ldp * 4);
    }
    L.bytes = off;
    return L;
}

int check_ce(const tig_softmax_ce *p)
{
    if (!p || p->struct_size != sizeof(tig_softmax_ce))
        return fail_text(TIG_EINVAL, "tig_softmax_ce: NULL argument or wrong struct_size");
    if (!dtype_ok(p->dtype) || p->reserved != 0)
        return fail_text(TIG_EINVAL, "tig_softmax_ce: unknown dtype, or reserved is not 0");
    if (p->rows < 0 || p->rows > (1 << 24) || p->vocab < 1 || p->vocab > (1 << 28) || p->dim < 1 || p->dim > (1 << 16))
        return fail_text(TIG_EINVAL, "tig_softmax_ce: rows, vocab or dim out of range");
    if (p->rows > 0 && (!p->x || !p->labels || !p->w))
        return fail_text(TIG_EINVAL, "tig_softmax_ce: x, w or labels is NULL");
    auto ld_ok = [&](int64_t ld) { return ld >= p->dim && ld <= (1 << 22); };
    if (!ld_ok(p->ldx) || !ld_ok(p->ldw) || (p->dx && !ld_ok(p->lddx)) || (p->dw && !ld_ok(p->lddw)))
        return fail_text(TIG_EINVAL, "tig_softmax_ce: a row stride is smaller than its row or above 2^22");
    auto aligned = [&](const void *q) { return (uintptr_t)q % (uintptr_t)dtype_bytes(p->dtype) == 0; };
    if (!aligned(p->x) || !aligned(p->w) || !aligned(p->bias) || !aligned(p->dx) || !aligned(p->dw) || !aligned(p->dbias) ||
        (((uintptr_t)p->labels | (uintptr_t)p->row_scale | (uintptr_t)p->loss | (uintptr_t)p->lse | (uintptr_t)p->mean) & 3))
        return fail_text(TIG_EINVAL, "tig_softmax_ce: an address is not aligned to its element");
    if (!(p->scale == p->scale) || p->scale - p->scale != 0.0f)
        return fail_text(TIG_EINVAL, "tig_softmax_ce: scale is not finite");
    return TIG_OK;
}

int check_ce_apart(const tig_softmax_ce &p)
{
    const int es = dtype_bytes(p.dtype);
    const int64_t n = p.rows, V = p.vocab, d = p.dim;
    const Placed in[] = {{p.x, n, d, p.ldx, es}, {p.w, V, d, p.ldw, es}, {p.bias, 1, V, V, es}, {n > 0 ? p.labels : nullptr, 1, n, n, 4},
                         {n > 0 ? p.row_scale : nullptr, 1, n, n, 4}};
    const Placed out[] = {{p.dx, n, d, p.lddx, es}, {p.dw, V, d, p.lddw, es}, {p.dbias, 1, V, V, es}, {n > 0 ? p.loss : nullptr, 1, n, n, 4},
                          {n > 0 ? p.lse : nullptr, 1, n, n, 4}, {p.mean, 1, 1, 1, 4}};
    return all_apart(in, out) ? TIG_OK : fail_text(TIG_EINVAL, "tig_softmax_ce: an output overlaps another tensor of the call");
}

#define CE_TRY(call)                 \
    do {                             \
        const hipError_t e_ = call;  \
        if (e_ != hipSuccess)        \
            return e_;               \
    } while (0)

template <typename T>
hipError_t launch_rows(const tig_softmax_ce &p, int64_t r, int64_t m, const float2 *part, int64_t tiles, const T *x, int64_t ldx, const T *w, int64_t ldw,
                       const CeHead *head, const CeRowsOut<T> &out, hipStream_t s)
{
    const int64_t all = out.lse2 ? (m + kNarrowStream - 1) / kNarrowStream * kNarrowStream : m;
    // (a wavefront a row where the parts of 16 lanes would be long chains of loads: 103 rows of 2165 tiles 63 us with 16, 14 with 64)
    const bool wide = tiles > 128 && m < 4096;
    hipLaunchKernelGGL((wide ? k_ce_rows<T, 64> : k_ce_rows<T, 16>), dim3((unsigned)(wide ? (all + 3) / 4 : (all + 15) / 16)), dim3(256), 0, s, part, tiles, m,
                       x + r * ldx, ldx, w, ldw, (const T *)p.bias, p.dim, p.vocab, p.labels + r, p.row_scale ? p.row_scale + r : nullptr, p.scale, head, out);
    return hipGetLastError();
}

hipError_t launch_mean(const tig_softmax_ce &p, const float *loss, const float *lse2, CeHead *head, hipStream_t s)
{
    hipLaunchKernelGGL(k_ce_mean, dim3(1), dim3(1024), 0, s, loss, p.labels, p.rows, p.vocab, p.row_scale != nullptr, p.scale, lse2, head, p.mean);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_copy(const T *src, int64_t ld_src, int64_t rows, int64_t cols, const T *extra, float fill, float behind, T *dst, int64_t ld_dst,
                       int64_t all, hipStream_t s)
{
    const int64_t blocks = (all * (ld_dst / Mat<T>::kPer16) + 255) / 256;
    hipLaunchKernelGGL((k_ce_copy<T>), dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, src, ld_src, rows, cols, extra, fill, behind, dst,
                       ld_dst, all);
    return hipGetLastError();
}

// 16-bit rows of at most 32 times KB columns; x and w are rows of whole 16-byte pieces
template <typename T, int KB, int DT, bool BIASED>
hipError_t run_narrow(const tig_softmax_ce &p, const CePlan &L, char *ws, const T *x, int64_t ldx, const T *w, int64_t ldw, const CeRowsOut<T> &out,
                      hipStream_t s)
{
    const int64_t n = p.rows, V = p.vocab;
    CeHead *const head = (CeHead *)(ws + L.head);
    const float alpha = 1.0f / kPScale<T>;
    float *bias32 = nullptr;
    if (p.bias && !BIASED) {
        bias32 = (float *)(ws + L.bias32);
        const int64_t all = L.cand_tiles * kNarrowStream;
        hipLaunchKernelGGL((k_ce_bias<T>), dim3((unsigned)((all + 255) / 256)), dim3(256), 0, s, (const T *)p.bias, V, bias32, all);
        CE_TRY(hipGetLastError());
    }
    const dim3 threads(64 * kNarrowWaves);
    NarrowArgs<T> a = {};
    a.own = x, a.ld_own = ldx, a.n_own = n;
    a.stream = w, a.ld_stream = ldw, a.n_stream = BIASED ? L.cand_tiles * kNarrowStream : V;
    a.d = (int)p.dim, a.k = a.d + (BIASED ? 1 : 0);
    a.stream_add = bias32;
    a.splits = L.s_stat, a.per = (L.cand_tiles + L.s_stat - 1) / L.s_stat;
    a.part = (float2 *)(ws + L.part);
    hipLaunchKernelGGL((k_narrow_stats<T, KB, BIASED>), dim3((unsigned)(L.own_rows * L.s_stat)), threads, 0, s, a);
    CE_TRY(hipGetLastError());
    CE_TRY(launch_rows(p, 0, n, a.part, L.s_stat, x, ldx, w, ldw, head, out, s));
    CE_TRY(launch_mean(p, out.loss, out.lse2, head, s));
    if (!L.grad)
        return hipSuccess;
    a.own = out.x0, a.ld_own = out.ld_x0;
    a.ld_grad = L.ld_acc;
    a.p_scale = kPScale<T>;
    a.lse2 = out.lse2, a.top = out.top, a.per_sum = out.per_sum, a.some_far = &head->some_far;
    if (p.dx) {
        a.splits = L.s_dx, a.per = (L.cand_tiles + L.s_dx - 1) / L.s_dx;
        a.labels = out.label;
        a.grad = (float *)(ws + L.dxa);
        hipLaunchKernelGGL((k_narrow_grad<T, KB, DT, BIASED, false, false>), dim3((unsigned)(L.own_rows * L.s_dx)), threads, 0, s, a);
        CE_TRY(hipGetLastError());
        const int64_t blocks = (n * ((p.dim + 3) / 4) + 255) / 256;
        hipLaunchKernelGGL((k_ce_narrow_dx<T>), dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, a.grad, L.s_dx, a.ld_grad, n, p.dim,
                           out.w, head, alpha, (T *)p.dx, p.lddx);
        CE_TRY(hipGetLastError());
    }
    if (p.dw || p.dbias) {
        a.own = w, a.ld_own = ldw, a.n_own = V;
        a.stream = out.x0, a.ld_stream = out.ld_x0, a.n_stream = BIASED ? L.row_tiles * kNarrowStream : n;
        a.own_add = bias32, a.stream_add = nullptr;
        a.w_stream = out.w, a.labels = out.label;
        a.splits = L.s_dw, a.per = (L.row_tiles + L.s_dw - 1) / L.s_dw;
        a.grad = p.dw && L.s_dw > 1 ? (float *)(ws + L.join) : nullptr;
        a.sums = p.dbias ? (float *)(ws + L.sums) : nullptr;
        const EpiStore<T> store = {(T *)p.dw, p.lddw, &head->S, alpha};
        if (p.dw && L.s_dw == 1)
            a.direct = store;
        const dim3 grid((unsigned)(L.own_cands * L.s_dw));
        if (p.row_scale || p.scale < 0.0f)
            hipLaunchKernelGGL((k_narrow_grad<T, KB, DT, BIASED, true, true>), grid, threads, 0, s, a);
        else
            hipLaunchKernelGGL((k_narrow_grad<T, KB, DT, BIASED, true, false>), grid, threads, 0, s, a);
        CE_TRY(hipGetLastError());
        if (p.dw && L.s_dw > 1)
            CE_TRY(launch_join(a.grad, L.s_dw, V, p.dim, a.ld_grad, store, s));
        if (p.dbias)
            CE_TRY((launch_join_sums<T>(a.sums, V, L.s_dw, V, (T *)p.dbias, &head->S, alpha, s)));
    }
    return hipSuccess;
}

template <typename T, bool BIASED>
hipError_t run_narrow_of(const tig_softmax_ce &p, const CePlan &L, char *ws, const T *x, int64_t ldx, const T *w, int64_t ldw, const CeRowsOut<T> &out,
                         hipStream_t s)
{
    if (p.dim <= 32)
        return run_narrow<T, 2, 2, BIASED>(p, L, ws, x, ldx, w, ldw, out, s);
    if (p.dim <= 64)
        return run_narrow<T, 2, 4, BIASED>(p, L, ws, x, ldx, w, ldw, out, s);
    if (p.dim <= 96)
        return run_narrow<T, 4, 6, BIASED>(p, L, ws, x, ldx, w, ldw, out, s);
    if (p.dim <= 112)
        return run_narrow<T, 4, 7, BIASED>(p, L, ws, x, ldx, w, ldw, out, s);
    return run_narrow<T, 4, 8, BIASED>(p, L, ws, x, ldx, w, ldw, out, s);
}

template <typename T>
hipError_t run(const tig_softmax_ce &p, const CePlan &L, char *ws, hipStream_t s)
{
    constexpr int es = sizeof(T);
    const int64_t n = p.rows, V = p.vocab, d = p.dim;
    CeHead *const head = (CeHead *)(ws + L.head);
    if (n == 0) {
        if (p.mean)
            CE_TRY(launch_zero_rows(p.mean, 1, 1, 1, 4, s));
        if (p.dw)
            CE_TRY(launch_zero_rows(p.dw, p.lddw, V, d, es, s));
        if (p.dbias)
            CE_TRY(launch_zero_rows(p.dbias, V, 1, V, es, s));
        return hipSuccess;
    }
    const T *x = (const T *)p.x, *w = (const T *)p.w, *bias = (const T *)p.bias;
    int64_t ldx = p.ldx, ldw = p.ldw;
    if (p.row_scale && L.grad) {
        hipLaunchKernelGGL(k_ce_top, dim3(1), dim3(1024), 0, s, p.labels, p.row_scale, p.scale, n, V, head);
        CE_TRY(hipGetLastError());
    }
    if (L.biased) {
        CE_TRY(launch_copy<T>(x, ldx, n, d, nullptr, 1.0f, 1.0f, (T *)(ws + L.px), L.ld_x, n, s));
        CE_TRY(launch_copy<T>(w, ldw, V, d, bias, 0.0f, -INFINITY, (T *)(ws + L.pw), L.ld_w, L.cand_tiles * kNarrowStream, s));
    } else {
        if (L.pack_x)
            CE_TRY(launch_pack(x, ldx, ws + L.px, L.ld_x, n, d, es, s));
        if (L.pack_w)
            CE_TRY(launch_pack(w, ldw, ws + L.pw, L.ld_w, V, d, es, s));
    }
    if (L.pack_x)
        x = (const T *)(ws + L.px), ldx = L.ld_x;
    if (L.pack_w)
        w = (const T *)(ws + L.pw), ldw = L.ld_w;
    float *const loss = p.loss ? p.loss : (float *)(ws + L.loss);
    CeRowsOut<T> out = {};
    out.loss = loss, out.lse = p.lse;
    if (L.grad && L.kb)
        out.lse2 = (float *)(ws + L.lse2), out.top = (float *)(ws + L.top), out.per_sum = (float *)(ws + L.per_sum), out.w = (float *)(ws + L.weight), out.label = (int32_t *)(ws + L.label);
    else if (L.grad)
        out.rec = (CeRow *)(ws + L.rec);
    if (L.grad && (L.kb || p.dw))
        out.x0 = (T *)(ws + L.px0), out.ld_x0 = L.ld_x, out.ones = L.biased;
    if constexpr (es == 2)
        if (L.kb)
            return L.biased ? run_narrow_of<T, true>(p, L, ws, x, ldx, w, ldw, out, s) : run_narrow_of<T, false>(p, L, ws, x, ldx, w, ldw, out, s);
    float2 *const part = (float2 *)(ws + L.part);
    const int64_t tiles = (V + L.stat.tile - 1) / L.stat.tile;
    for (int64_t r = 0; r < n; r += L.stat_rows) {
        const int64_t m = n - r < L.stat_rows ? n - r : L.stat_rows;
        const EpiStats<T> epi = {bias, part, m};
        CE_TRY((launch_gemm<T, kRow, kRow>(L.stat, x + r * ldx, ldx, w, ldw, m, V, d, nullptr, epi, s)));
        CeRowsOut<T> o = out;
        o.loss += r;
        o.lse = o.lse ? o.lse + r : nullptr;
        o.rec = o.rec ? o.rec + r : nullptr;
        o.x0 = o.x0 ? o.x0 + r * o.ld_x0 : nullptr;
        CE_TRY(launch_rows(p, r, m, part, tiles, x, ldx, w, ldw, head, o, s));
    }
    CE_TRY(launch_mean(p, loss, nullptr, head, s));
    if (!L.grad)
        return hipSuccess;
    const float alpha = 1.0f / kPScale<T>;
    T *const P = (T *)(ws + L.P);
    for (int64_t v0 = 0; v0 < V; v0 += L.piece) {
        const int64_t vc = V - v0 < L.piece ? V - v0 : L.piece;
        float *const sums = p.dbias ? (float *)(ws + L.sums) : nullptr;
        const EpiP<T> epi = {bias ? bias + v0 : nullptr, out.rec, P, L.ldp, v0, sums};
        CE_TRY((launch_gemm<T, kRow, kRow>(L.logits, x, ldx, w + v0 * ldw, ldw, n, vc, d, nullptr, epi, s)));
        if (p.dbias)
            CE_TRY((launch_join_sums<T>(sums, L.ldp, (n + L.logits.tile - 1) / L.logits.tile, vc, (T *)p.dbias + v0, &head->S, alpha, s)));
        if (p.dx) {
            if (L.acc) {
                const EpiAdd add = {(float *)(ws + L.dxa), L.ld_acc, v0 == 0};
                CE_TRY((launch_gemm<T, kRow, kCol>(L.dx, P, L.ldp, w + v0 * ldw, ldw, n, d, vc, ws + L.join, add, s)));
            } else {
                const EpiStore<T> store = {(T *)p.dx, p.lddx, &head->S, alpha};
                CE_TRY((launch_gemm<T, kRow, kCol>(L.dx, P, L.ldp, w, ldw, n, d, vc, ws + L.join, store, s)));
            }
        }
        if (p.dw) {
            T *const dw = (T *)p.dw + v0 * p.lddw;
            const EpiStore<T> store = {dw, p.lddw, &head->S, alpha};
            CE_TRY((launch_gemm<T, kCol, kCol>(L.dw, P, L.ldp, out.x0, L.ld_x, vc, d, n, ws + L.join, store, s)));
        }
    }
    if (p.dx && L.acc) {
        const int64_t blocks = (n * ((d + 3) / 4) + 255) / 256;
        hipLaunchKernelGGL((k_ce_dx<T>), dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, (const float *)(ws + L.dxa), L.ld_acc, n, d,
                           &head->S, alpha, (T *)p.dx, p.lddx);
        CE_TRY(hipGetLastError());
    }
    return hipSuccess;
}

}  // namespace

}  // namespace tig

using namespace tig;

int tig_softmax_ce_workspace_bytes(const tig_softmax_ce *p, size_t *bytes)
{
    const int rc = check_ce(p);
    if (rc != TIG_OK)
        return rc;
    if (!bytes)
        return fail_text(TIG_EINVAL, "tig_softmax_ce_workspace_bytes: bytes is NULL");
    *bytes = ce_plan(*p).bytes;
    return TIG_OK;
}

// For tests: does the call go the way of ce_narrow.h (1), or by tiles (0)?  -1: it is refused.
extern "C" __attribute__((visibility("default"))) int tig_debug_softmax_ce_narrow(const tig_softmax_ce *p)
{
    return check_ce(p) != TIG_OK ? -1 : ce_plan(*p).kb != 0;
}

int tig_softmax_ce_run(const tig_softmax_ce *p, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_ce(p);
    if (rc != TIG_OK)
        return rc;
    if (!workspace || ((uintptr_t)workspace & 255))
        return fail_text(TIG_EINVAL, "tig_softmax_ce_run: workspace is NULL or not 256-byte aligned");
    const CePlan L = ce_plan(*p);
    if (workspace_bytes < L.bytes)
        return fail_text(TIG_ENOSPACE, "tig_softmax_ce_run: workspace too small");
    if ((rc = check_ce_apart(*p)) != TIG_OK)
        return rc;
    const hipError_t e = with_dtype(p->dtype, [&](auto t) { return run<decltype(t)>(*p, L, (char *)workspace, (hipStream_t)hip_stream); });
    return e == hipSuccess ? TIG_OK : fail_global("tig_softmax_ce_run", e);
}
