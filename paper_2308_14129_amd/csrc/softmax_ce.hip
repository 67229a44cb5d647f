// Softmax cross entropy of rows over a vocabulary of candidates, with its gradient (include/tig.h, tig_softmax_ce_*).  gfx950.
//
//   statistics   a tile product X W^T (gemm.h) whose epilogue leaves, for every row and tile of candidates, the largest logit and
//                the sum of exp(l - largest); k_ce_rows joins them to the row's log-sum-exp and takes the label's logit
//   gradient     for one piece of the vocabulary after the other: the logits once more, P = w_i (exp(l - lse) - [label]) in their
//                epilogue, and two tile products, dX += P W and dW = P^T X.  A piece of P stays within the last-level cache.
// s_i = S w_i with S the largest |s_i|: P holds values of at most 1, the products are scaled by S afterwards.
#include "act.h"
#include "gemm.h"

namespace tig {

namespace {

struct CeHead {
    float S;         // largest |s_i|
    int32_t counted; // rows that count
};
// what the epilogue of P needs of a row: lse (+infinity: no probabilities) and w_i * P's scale
struct CeRow {
    float lse, w;
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

// number of rows that count and the largest |s_i|
__global__ void __launch_bounds__(1024) k_ce_head(const int32_t *labels, const float *row_scale, float scale, int64_t rows, int64_t vocab, CeHead *head)
{
    __shared__ int n_of[16];
    __shared__ float top_of[16];
    int n = 0;
    float top = 0.0f;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) {
        const int32_t label = labels[i];
        if (label >= 0 && label < vocab) {
            ++n;
            if (row_scale)
                top = fmaxf(top, fabsf(row_scale[i]));
        }
    }
    for (int d = 32; d > 0; d >>= 1) {
        n += __shfl_xor(n, d);
        top = fmaxf(top, __shfl_xor(top, d));
    }
    if (lane_id() == 0)
        n_of[wave_id()] = n, top_of[wave_id()] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) {
            n += n_of[w];
            top = fmaxf(top, top_of[w]);
        }
        head->counted = n;
        head->S = row_scale ? top * fabsf(scale) : fabsf(scale) / (float)(n > 0 ? n : 1);
    }
}

// Largest logit and sum of exponentials of a row over a tile of candidates: over a lane's columns, the four lanes of a row, and
// the wavefronts side by side (in LDS).  part[tile][row].
template <typename T>
struct EpiStats {
    static constexpr bool kWhole = true;
    const T *bias;
    bool bias_ok;
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
                b = load_four(bias + n, left, bias_ok);
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

// Sixteen rows per workgroup, sixteen threads each: the tiles' parts joined, the label's logit, loss.
template <typename T>
__global__ void __launch_bounds__(256) k_ce_rows(const float2 *part, int64_t tiles, int64_t rows, const T *x, int64_t ldx, const T *w, int64_t ldw,
                                                 const T *bias, int64_t dim, int64_t vocab, const int32_t *labels, const float *row_scale, float scale,
                                                 const CeHead *head, float *loss, float *lse_out, CeRow *rec, float *label_logit)
{
    const int64_t i = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const int t = threadIdx.x % 16;
    const bool on = i < rows;
    const int64_t r = on ? i : rows - 1;
    float top = -INFINITY, sum = 0.0f;
    for (int64_t k = t; k < tiles; k += 16) {
        const float2 v = part[k * rows + r];
        const float to = fmaxf(top, v.x), from = to == -INFINITY ? 0.0f : to;
        sum = sum * expf(top - from) + v.y * expf(v.x - from);
        top = to;
    }
    const int32_t label = labels[r];
    const bool counts = label >= 0 && label < vocab;
    float dot = 0.0f;
    const T *xr = x + r * ldx, *wr = w + (counts ? (int64_t)label : 0) * ldw;
    for (int64_t k = t; k < dim; k += 16)
        dot += to_float(xr[k]) * to_float(wr[k]);
    for (int d = 8; d > 0; d >>= 1) {
        const float ot = __shfl_xor(top, d), os = __shfl_xor(sum, d);
        const float to = fmaxf(top, ot), from = to == -INFINITY ? 0.0f : to;
        sum = sum * expf(top - from) + os * expf(ot - from);
        top = to;
        dot += __shfl_xor(dot, d);
    }
    if (!on || t != 0)
        return;
    const float lse = top == -INFINITY && sum == 0.0f ? -INFINITY : top + logf(sum);
    if (bias && counts)
        dot += to_float(bias[label]);
    if (lse_out)
        lse_out[i] = lse;
    if (loss)
        loss[i] = !counts ? 0.0f : (dot == -INFINITY ? INFINITY : lse - dot);
    if (rec) {
        float wi = 0.0f;
        if (counts)
            wi = row_scale ? (head->S > 0.0f ? row_scale[i] * scale / head->S : 0.0f) : (scale < 0.0f ? -1.0f : 1.0f);
        rec[i] = CeRow{wi != 0.0f && lse != -INFINITY ? lse : INFINITY, wi * kPScale<T>};
        label_logit[i] = dot;
    }
}

// P of a piece of the vocabulary, columns up to a whole 16-byte piece zero (the label's place: k_ce_labels)
template <typename T>
struct EpiP {
    static constexpr bool kWhole = false;
    const T *bias;
    bool bias_ok;
    const CeRow *rec;
    T *P;
    int64_t ldp;
    __device__ inline CeRow row(int64_t m) const { return rec[m]; }
    __device__ inline void operator()(const CeRow &r, int64_t m, int64_t n, floatx4 v, int left) const
    {
        if (bias)
            v += load_four(bias + n, left, bias_ok);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = e < left && r.lse != INFINITY ? exp_of<T>(v[e] - r.lse) * r.w : 0.0f;
        store_four(P + m * ldp + n, v, 4, true);
    }
};

// P at the labels of the piece [v0, v0 + vc), and the zeros behind its last column up to a whole 16-byte piece
template <typename T>
__global__ void __launch_bounds__(256) k_ce_labels(T *P, int64_t ldp, int64_t rows, int64_t v0, int64_t vc, const int32_t *labels, const CeRow *rec,
                                                   const float *label_logit)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows)
        return;
    constexpr int64_t per = Mat<T>::kPer16;
    for (int64_t c = (vc + 3) / 4 * 4; c < (vc + per - 1) / per * per; ++c)
        P[i * ldp + c] = (T)0.0f;
    const int64_t c = (int64_t)labels[i] - v0;
    const CeRow r = rec[i];
    if (c >= 0 && c < vc && r.w != 0.0f) {
        const float l = label_logit[i];
        const float p = r.lse == INFINITY || l == -INFINITY ? 0.0f : expf(l - r.lse);
        P[i * ldp + c] = (T)((p - 1.0f) * r.w);
    }
}

// a piece's share of dX: stored, or added to the pieces before it
struct EpiAdd {
    static constexpr bool kWhole = false;
    float *acc;
    int64_t ld;
    bool first;
    __device__ inline int row(int64_t) const { return 0; }
    __device__ inline void operator()(int, int64_t m, int64_t n, floatx4 v, int) const
    {
        floatx4 *const p = (floatx4 *)(acc + m * ld + n);
        *p = first ? v : *p + v;
    }
};

template <typename T>
__global__ void __launch_bounds__(256) k_ce_dx(const float *acc, int64_t ld, int64_t rows, int64_t dim, const float *scale, float alpha, T *dx,
                                               int64_t lddx, bool aligned)
{
    const int64_t per = (dim + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * per; i += (int64_t)gridDim.x * 256) {
        const int64_t m = i / per, n = i % per * 4;
        const floatx4 v = *(const floatx4 *)(acc + m * ld + n) * (alpha * *scale);
        store_four(dx + m * lddx + n, v, dim - n < 4 ? (int)(dim - n) : 4, aligned);
    }
}

// column sums of a piece of P over blocks of rows, eight columns per thread
constexpr int kSumRows = 64;
template <typename T>
__global__ void __launch_bounds__(256) k_ce_sums(const T *P, int64_t ldp, int64_t rows, int64_t vc, int64_t per, float *sums, int64_t lds)
{
    const int64_t n = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (n >= vc)
        return;
    const int64_t m0 = (int64_t)blockIdx.y * per, m1 = m0 + per < rows ? m0 + per : rows;
    floatx4 total = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int64_t m = m0; m < m1; ++m)
        total += load_four(P + m * ldp + n, 4, true);
    *(floatx4 *)(sums + (int64_t)blockIdx.y * lds + n) = total;
}

// mean of the rows that count, in double, always in the same order
__global__ void __launch_bounds__(1024) k_ce_mean(const float *loss, int64_t rows, const CeHead *head, float *mean)
{
    __shared__ double part[1024];
    double total = 0.0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024)
        total += (double)loss[i];
    part[threadIdx.x] = total;
    __syncthreads();
    for (int d = 512; d > 0; d >>= 1) {
        if ((int)threadIdx.x < d)
            part[threadIdx.x] += part[threadIdx.x + d];
        __syncthreads();
    }
    if (threadIdx.x == 0)
        *mean = (float)(part[0] / (double)(head && head->counted > 0 ? head->counted : 1));
}

inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct CePlan {
    bool grad, pack_x, pack_w;
    int64_t ld_x, ld_w;      // of the packed copies
    int64_t stat_rows;       // rows whose statistics are formed at a time
    GemmPlan stat;
    int64_t piece;           // candidates of a piece
    GemmPlan logits, dx, dw;
    int64_t ldp, ld_acc, sum_per, sum_blocks;
    bool acc;                // more than one piece: dX in fp32 first
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
        L.label = take(4 * (size_t)n);
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
        L.sum_per = n <= (int64_t)kSumRows * 32768 ? kSumRows : (n + 32767) / 32768;
        L.sum_blocks = (n + L.sum_per - 1) / L.sum_per;
        if (p.dbias)
            L.sums = take((size_t)L.sum_blocks * L.ldp * 4);
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
    if (p->rows < 0 || p->rows > (1 << 24) || p->vocab < 1 || p->vocab > 0x7fffffff || p->dim < 1 || p->dim > (1 << 16))
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

#define CE_TRY(call)                 \
    do {                             \
        const hipError_t e_ = call;  \
        if (e_ != hipSuccess)        \
            return e_;               \
    } while (0)

template <typename T>
hipError_t run(const tig_softmax_ce &p, const CePlan &L, char *ws, hipStream_t s)
{
    const int es = sizeof(T);
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
    hipLaunchKernelGGL(k_ce_head, dim3(1), dim3(1024), 0, s, p.labels, p.row_scale, p.scale, n, V, head);
    CE_TRY(hipGetLastError());
    if (L.pack_x) {
        CE_TRY(launch_pack(x, ldx, ws + L.px, L.ld_x, n, d, es, nullptr, s));
        x = (const T *)(ws + L.px), ldx = L.ld_x;
    }
    if (L.pack_w) {
        CE_TRY(launch_pack(w, ldw, ws + L.pw, L.ld_w, V, d, es, nullptr, s));
        w = (const T *)(ws + L.pw), ldw = L.ld_w;
    }
    const bool bias_ok = four_aligned(bias, 4, es);
    float *const loss = p.loss ? p.loss : (float *)(ws + L.loss);
    CeRow *const rec = L.grad ? (CeRow *)(ws + L.rec) : nullptr;
    float *const label = L.grad ? (float *)(ws + L.label) : nullptr;
    float2 *const part = (float2 *)(ws + L.part);
    const int64_t tiles = (V + L.stat.tile - 1) / L.stat.tile;
    for (int64_t r = 0; r < n; r += L.stat_rows) {
        const int64_t m = n - r < L.stat_rows ? n - r : L.stat_rows;
        const EpiStats<T> epi = {bias, bias_ok, part, m};
        CE_TRY((launch_gemm<T, kRow, kRow>(L.stat, x + r * ldx, ldx, w, ldw, m, V, d, nullptr, epi, s)));
        hipLaunchKernelGGL((k_ce_rows<T>), dim3((unsigned)((m + 15) / 16)), dim3(256), 0, s, part, tiles, m, x + r * ldx, ldx, w, ldw, bias, d, V,
                           p.labels + r, p.row_scale ? p.row_scale + r : nullptr, p.scale, head, loss + r, p.lse ? p.lse + r : nullptr,
                           rec ? rec + r : nullptr, label ? label + r : nullptr);
        CE_TRY(hipGetLastError());
    }
    if (p.mean) {
        hipLaunchKernelGGL(k_ce_mean, dim3(1), dim3(1024), 0, s, loss, n, head, p.mean);
        CE_TRY(hipGetLastError());
    }
    if (!L.grad)
        return hipSuccess;
    const float alpha = 1.0f / kPScale<T>;
    T *const P = (T *)(ws + L.P);
    const T *x0 = nullptr;  // rows that do not count as zeros: whatever they hold, P^T X does not see it
    if (p.dw) {
        CE_TRY(launch_pack(x, ldx, ws + L.px0, L.ld_x, n, d, es, &rec->w, s));
        x0 = (const T *)(ws + L.px0);
    }
    for (int64_t v0 = 0; v0 < V; v0 += L.piece) {
        const int64_t vc = V - v0 < L.piece ? V - v0 : L.piece;
        const EpiP<T> epi = {bias ? bias + v0 : nullptr, bias && four_aligned(bias + v0, 4, es), rec, P, L.ldp};
        CE_TRY((launch_gemm<T, kRow, kRow>(L.logits, x, ldx, w + v0 * ldw, ldw, n, vc, d, nullptr, epi, s)));
        hipLaunchKernelGGL((k_ce_labels<T>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, P, L.ldp, n, v0, vc, p.labels, rec, label);
        CE_TRY(hipGetLastError());
        if (p.dbias) {
            hipLaunchKernelGGL((k_ce_sums<T>), dim3((unsigned)((vc + 1023) / 1024), (unsigned)L.sum_blocks), dim3(256), 0, s, P, L.ldp, n, vc, L.sum_per,
                               (float *)(ws + L.sums), L.ldp);
            CE_TRY(hipGetLastError());
            CE_TRY((launch_join_sums<T>((const float *)(ws + L.sums), L.ldp, L.sum_blocks, vc, (T *)p.dbias + v0, &head->S, alpha, s)));
        }
        if (p.dx) {
            if (L.acc) {
                const EpiAdd add = {(float *)(ws + L.dxa), L.ld_acc, v0 == 0};
                CE_TRY((launch_gemm<T, kRow, kCol>(L.dx, P, L.ldp, w + v0 * ldw, ldw, n, d, vc, ws + L.join, add, s)));
            } else {
                const EpiStore<T> out = {(T *)p.dx, p.lddx, &head->S, alpha, four_aligned(p.dx, p.lddx, es)};
                CE_TRY((launch_gemm<T, kRow, kCol>(L.dx, P, L.ldp, w, ldw, n, d, vc, ws + L.join, out, s)));
            }
        }
        if (p.dw) {
            T *const dw = (T *)p.dw + v0 * p.lddw;
            const EpiStore<T> out = {dw, p.lddw, &head->S, alpha, four_aligned(dw, p.lddw, es)};
            CE_TRY((launch_gemm<T, kCol, kCol>(L.dw, P, L.ldp, x0, L.ld_x, vc, d, n, ws + L.join, out, s)));
        }
    }
    if (p.dx && L.acc) {
        const int64_t blocks = (n * ((d + 3) / 4) + 255) / 256;
        hipLaunchKernelGGL((k_ce_dx<T>), dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, (const float *)(ws + L.dxa), L.ld_acc, n, d,
                           &head->S, alpha, (T *)p.dx, p.lddx, four_aligned(p.dx, p.lddx, es));
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

int tig_softmax_ce_run(const tig_softmax_ce *p, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const int rc = check_ce(p);
    if (rc != TIG_OK)
        return rc;
    if (!workspace || ((uintptr_t)workspace & 255))
        return fail_text(TIG_EINVAL, "tig_softmax_ce_run: workspace is NULL or not 256-byte aligned");
    const CePlan L = ce_plan(*p);
    if (workspace_bytes < L.bytes)
        return fail_text(TIG_ENOSPACE, "tig_softmax_ce_run: workspace too small");
    const hipError_t e = with_dtype(p->dtype, [&](auto t) { return run<decltype(t)>(*p, L, (char *)workspace, (hipStream_t)hip_stream); });
    return e == hipSuccess ? TIG_OK : fail_global("tig_softmax_ce_run", e);
}
