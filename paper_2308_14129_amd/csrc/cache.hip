// Paged key-value cache (include/tig.h): what is common, new tokens (tig_cache_append), and sequences that are taken over by
// several others (tig_cache_fork).  gfx950.
#include "cache.h"

namespace tig {

Placed placed(const void *p, std::initializer_list<Dim> dims, int64_t cols, int elem)
{
    Dim d[3] = {};
    int n = 0;
    for (const Dim &x : dims)
        if (x.n > 1)
            d[n++] = x;
    std::sort(d, d + n, [](const Dim &a, const Dim &b) { return a.stride > b.stride; });
    while (n > 1 && d[0].stride == d[1].n * d[1].stride) {
        d[1].n *= d[0].n;
        for (int i = 1; i < n; ++i)
            d[i - 1] = d[i];
        --n;
    }
    for (int i = 1; i < n; ++i)
        cols += (d[i].n - 1) * d[i].stride;
    if (n == 0)
        return {p, 1, cols, cols, elem};
    if (cols > d[0].stride)  // not rows: one range
        return {p, 1, cols + (d[0].n - 1) * d[0].stride, cols, elem};
    return {p, d[0].n, cols, d[0].stride, elem};
}

bool rows_meet(int64_t n_a, int64_t stride_a, int64_t n_b, int64_t stride_b, int64_t cols)
{
    if ((n_a > 1 && stride_a < cols) || (n_b > 1 && stride_b < cols))
        return true;
    if (n_a <= 1 || n_b <= 1 || stride_a >= (n_b - 1) * stride_b + cols || stride_b >= (n_a - 1) * stride_a + cols)
        return false;
    if (n_a < n_b)
        std::swap(n_a, n_b), std::swap(stride_a, stride_b);
    for (int64_t j = 1; j < n_b; ++j) {  // j steps of the one against the steps of the other on both sides of them (of heads there are 2^14 at most)
        const int64_t i = j * stride_b / stride_a, past = j * stride_b - i * stride_a;
        if ((i > 0 && i < n_a && past < cols) || (i + 1 < n_a && stride_a - past < cols))
            return true;
    }
    return false;
}

int check_cache(const tig_cache *c)
{
    if (!c || c->struct_size != sizeof(tig_cache))
        return fail_text(TIG_EINVAL, "tig_cache: NULL argument or wrong struct_size");
    if (!dtype_ok(c->dtype))
        return fail_text(TIG_EINVAL, "tig_cache: unknown dtype");
    if (c->pages < 1 || c->pages > 0x7fffffff || c->page_size < 1 || c->page_size > (1 << 16) || c->heads < 1 || c->heads > (1 << 10) || c->head_dim < 8 ||
        c->head_dim > 256 || c->max_pages < 1 || c->max_pages > (1 << 24) || (int64_t)c->max_pages * c->page_size > 0x7fff0000)
        return fail_text(TIG_EINVAL, "tig_cache: pages, page_size, heads, head_dim or max_pages out of range");
    const int es = dtype_bytes(c->dtype);
    if (!c->k || !c->v || !element_aligned(c->k, es) || !element_aligned(c->v, es))
        return fail_text(TIG_EINVAL, "tig_cache: k or v is NULL or not aligned to its element");
    const int64_t most = (int64_t)1 << 40;
    if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0 || c->page_stride > most || c->token_stride > most || c->head_stride > most ||
        c->token_stride > 0x7fffffff || (c->page_size > 1 && c->page_size * c->token_stride * es > (1 << 30)))
        return fail_text(TIG_EINVAL, "tig_cache: a stride is out of range");
    if ((int64_t)c->page_size * c->heads * c->head_dim * es > (1 << 30))
        return fail_text(TIG_EINVAL, "tig_cache: a page is larger than 1 GiB");
    Dim d[3] = {{c->pages, c->page_stride}, {c->page_size, c->token_stride}, {c->heads, c->head_stride}};
    std::sort(d, d + 3, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
    int64_t span = c->head_dim;
    for (const Dim &x : d) {
        if (x.n > 1 && x.stride < span)
            return fail_text(TIG_EINVAL, "tig_cache: pages, rows and heads overlap");
        span += (x.n - 1) * x.stride;
        if (x.n > 1 && span > ((int64_t)1 << 46))
            return fail_text(TIG_EINVAL, "tig_cache: a stride is out of range");
    }
    return TIG_OK;
}

int check_sequences(const tig_cache &c, int64_t seqs, const int32_t *table, int64_t ld, const int32_t *lengths)
{
    if (seqs < 0 || seqs > (1 << 20))
        return fail_text(TIG_EINVAL, "tig_cache: number of sequences out of range");
    if (seqs > 0 && (!table || !lengths || !element_aligned(table, 4) || !element_aligned(lengths, 4)))
        return fail_text(TIG_EINVAL, "tig_cache: table or lengths is NULL or not aligned to its element");
    if (ld < c.max_pages || ld > ((int64_t)1 << 32))
        return fail_text(TIG_EINVAL, "tig_cache: the table's row stride is smaller than max_pages or above 2^32");
    return TIG_OK;
}

namespace {

// ------------------------------------------------------------------------------------------
// New tokens.

struct AppendArgs {
    CacheView c;
    int64_t seqs, tokens;
    const int32_t *starts;
    const void *positions;
    const double *freq;
    const char *k, *v, *q;
    char *qo;
    int64_t k_token, k_head, v_token, v_head, q_token, q_head, qo_token, qo_head;  // bytes
    int32_t q_heads, rotary, interleaved, position_type;
};

constexpr double kTurn8 = 0.63661977236758134308;  // 2 / pi
// pi / 2 in two parts
constexpr double kQuarterHi = 1.57079632679489655800, kQuarterLo = 6.12323399573676603587e-17;

// Cosine and sine of an angle in fp64: quarter turns are taken off (exactly, by fused products with the two parts of pi / 2), the rest, at
// most pi / 4, goes through the Taylor polynomials to the thirteenth and twelfth degree (their next terms are 2e-14 and 4e-13 there), and
// each is rounded once.  About 30 operations at fp64's rate, which is fp32's on this card.
// Of a far angle the first count n is off by up to 2^-52 of itself, so that a second one is taken off what is left.  The two stay apart: only
// their last two bits are wanted, and their sum would be rounded where n is beyond 2^53.  Up to 2^64 n is off by up to 2^12, what is
// left is 2^13 at most, and rounding that (2^-40), and what pi / 2 is beyond its two parts (n times 1.5e-33), come to less than 1e-11.
constexpr double kFarthest = 18446744073709551616.0;
__device__ inline void cos_sin(double angle, float &c, float &s)
{
    const double n = rint(angle * kTurn8);
    double x = fma(n, -kQuarterHi, angle);
    x = fma(n, -kQuarterLo, x);
    const double again = rint(x * kTurn8);
    x = fma(again, -kQuarterHi, x);
    if (!(fabs(angle) <= kFarthest))
        x = NAN;
    const double y = x * x;
    double ps = 1.0 / 6227020800.0, pc = 1.0 / 479001600.0;
    ps = fma(y, ps, -1.0 / 39916800.0);
    ps = fma(y, ps, 1.0 / 362880.0);
    ps = fma(y, ps, -1.0 / 5040.0);
    ps = fma(y, ps, 1.0 / 120.0);
    ps = fma(y, ps, -1.0 / 6.0);
    ps = fma(x * y, ps, x);
    pc = fma(y, pc, -1.0 / 3628800.0);
    pc = fma(y, pc, 1.0 / 40320.0);
    pc = fma(y, pc, -1.0 / 720.0);
    pc = fma(y, pc, 1.0 / 24.0);
    pc = fma(y, pc, -0.5);
    pc = fma(y, pc, 1.0);
    const int quarter = ((int)(n - 4.0 * floor(n * 0.25)) + (int)again) & 3;
    const double a = quarter & 1 ? ps : pc, b = quarter & 1 ? pc : ps;
    c = (float)((quarter + 1) & 2 ? -a : a);
    s = (float)(quarter & 2 ? -b : b);
}

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Piece16 {
    T v[16 / sizeof(T)];
};

// a' = a cos - b sin, b' = b cos + a sin for `n` pairs
template <typename T>
__device__ inline void rotate_pair(T &a, T &b, float c, float s)
{
    const float x = to_float(a), y = to_float(b);
    a = (T)fmaf(x, c, -(y * s));
    b = (T)fmaf(y, c, x * s);
}

// A workgroup takes `per` tokens: where each goes, the cosines and sines of its pairs (once for all its heads, in LDS), then the rows in
// units of 16 bytes, a rotated pair of pieces to a lane.  A lane has the same unit of every token (or of every `groups`-th one, where a token
// has few): what it has to divide it divides once, and the pieces of several tokens are on their way together.
constexpr int kAppendTokens = 16;

constexpr int kAppendDeep = 4;  // tokens whose pieces are on their way together

// Units of a row (pairs of pieces, pieces behind them, pieces of v), of all rows (`turning`, `resting`, `all`); tokens at a time, tokens of
// a workgroup.
struct AppendUnits {
    int32_t n_pair, n_rest, n_v, turning, resting, all, groups, per, in_place, shift;
};

struct AppendShared {
    float turn[kAppendTokens][2][128];  // cosines, sines
    int64_t at[kAppendTokens];          // the row's first byte, head 0; -1: none
    double position[kAppendTokens];
};

// where the workgroup's tokens go, and their cosines and sines
__device__ inline void append_places(const AppendArgs &a, int64_t token0, int count, AppendShared &sh)
{
    const CacheView &c = a.c;
    const int tid = threadIdx.x, pairs = a.rotary / 2;
    if (tid < count) {
        const int64_t token = token0 + tid;
        int64_t seq = token, row = -1;
        int place = -1;
        if (a.starts) {  // the last sequence that starts at or before the token
            int64_t lo = 0, hi = a.seqs;
            while (lo < hi) {
                const int64_t mid = (lo + hi + 1) / 2;
                if (a.starts[mid] <= token)
                    lo = mid;
                else
                    hi = mid - 1;
            }
            seq = lo;
            if (seq < a.seqs && a.starts[seq] <= token && token < a.starts[seq + 1])
                place = (int)std::max<int64_t>(c.lengths[seq] - (a.starts[seq + 1] - token), -1);
        } else {
            place = std::max(c.lengths[seq], 0) - 1;
        }
        if (place >= 0 && place < c.capacity()) {
            const int in_table = c.div.quotient(place), page = c.table[seq * c.ld_table + in_table];
            if (c.page_ok(page))
                row = c.offset(page, place - in_table * c.page_size, 0);
        }
        sh.at[tid] = row;
        sh.position[tid] = a.position_type == 0 ? (double)place : a.position_type == 1 ? (double)((const int64_t *)a.positions)[token]
                                                                                     : ((const double *)a.positions)[token];
    }
    __syncthreads();
    for (int i = tid; i < count * pairs; i += 256) {
        const int t = i / pairs, j = i - t * pairs;
        cos_sin(sh.position[t] * a.freq[j], sh.turn[t][0][j], sh.turn[t][1][j]);
    }
    __syncthreads();
}

// Rows by pieces of 16 bytes: a lane has one piece of a row and, for the pairs' other halves, reads the piece that lies there as well (it
// is on its way for another lane of the wavefront), so that reads and writes are whole lines: with a pair of pieces to a lane 62500 tokens of
// 40 rows of 256 bytes, 192 of them turned, took 347 us, so they take 260 (a copy of as much 250).  Rows do not cross wavefronts: one
// may be turned in place.  IN_PLACE: queries are; their lanes' reads then come before their lanes' writes for the compiler too, which else has some
// tokens' loads behind others' stores (the same prompts: 260 us, with that order 264).
template <typename T, bool IN_PLACE>
__global__ void __launch_bounds__(256) k_cache_append_rows(AppendArgs a, AppendUnits n)
{
    constexpr int VE = 16 / sizeof(T), ES = sizeof(T);
    __shared__ AppendShared sh;
    const int tid = threadIdx.x;
    const int64_t token0 = (int64_t)blockIdx.x * n.per;
    const int count = (int)std::min<int64_t>(n.per, a.tokens - token0);
    const CacheView &c = a.c;
    const int pairs = a.rotary / 2;
    append_places(a, token0, count, sh);
    for (int u = blockIdx.y * 256 + tid; u < n.all; u += 256 * gridDim.y) {
        const int r = u >> n.shift, w = u & ((1 << n.shift) - 1);
        const char *from;
        char *to;
        int64_t from_token, to_token = -1;
        const bool is_q = r < a.q_heads, is_k = !is_q && r < a.q_heads + c.heads;
        if (is_q) {
            from = a.q + r * a.q_head, from_token = a.q_token;
            to = a.qo + r * a.qo_head, to_token = a.qo_token;
        } else if (is_k) {
            from = a.k + (r - a.q_heads) * a.k_head, from_token = a.k_token;
            to = c.k + (r - a.q_heads) * c.head_stride;
        } else {
            from = a.v + (r - a.q_heads - c.heads) * a.v_head, from_token = a.v_token;
            to = c.v + (r - a.q_heads - c.heads) * c.head_stride;
        }
        // the piece's first column: pieces of each part of the row (halves of the pairs, or the pairs; what is behind them), the last of a
        // part from its end (some columns twice, from the same values: all lanes of the row have read before one writes)
        const int parts = a.interleaved ? 1 : 2, turned = is_q || is_k ? parts * n.n_pair : 0;
        const bool turns = w < turned, first = w < n.n_pair;
        const int begin = !turns ? (turned > 0 ? a.rotary : 0) : first ? 0 : pairs, end = !turns ? c.head_dim : a.interleaved ? a.rotary : first ? pairs : a.rotary;
        const int at = begin + (w - (!turns ? turned : first ? 0 : n.n_pair)) * VE, e = std::min(at, end - VE);
        if (at >= end)
            continue;
        const int other = !turns || a.interleaved ? e : first ? e + pairs : e - pairs;
        const int j = a.interleaved ? e / 2 : first ? e : e - pairs;
        from += token0 * from_token;
        for (int t0 = 0; t0 < count; t0 += kAppendDeep) {
            Piece16<T> x[kAppendDeep], y[kAppendDeep];
#pragma unroll
            for (int i = 0; i < kAppendDeep; ++i) {
                const char *const p = from + std::min(t0 + i, count - 1) * from_token;
                x[i] = *(const Piece16<T> *)(p + e * ES);
                y[i] = *(const Piece16<T> *)(p + other * ES);
            }
            if constexpr (IN_PLACE) {
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "global");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "global");
            }
#pragma unroll
            for (int i = 0; i < kAppendDeep; ++i) {
                const int t = t0 + i;
                if (t >= count || sh.at[t] < 0)
                    continue;
                if (turns) {
                    const float *const cs = sh.turn[t][0] + j, *const sn = sh.turn[t][1] + j;
                    if (a.interleaved) {
#pragma unroll
                        for (int k = 0; k < VE / 2; ++k)
                            rotate_pair(x[i].v[2 * k], x[i].v[2 * k + 1], cs[k], sn[k]);
                    } else {
#pragma unroll
                        for (int k = 0; k < VE; ++k) {
                            const float s = to_float(y[i].v[k]) * sn[k];
                            x[i].v[k] = (T)fmaf(to_float(x[i].v[k]), cs[k], first ? -s : s);
                        }
                    }
                }
                *(Piece16<T> *)(to + (to_token < 0 ? sh.at[t] : (token0 + t) * to_token) + e * ES) = x[i];
            }
        }
    }
}

// Rows with a part that is shorter than a piece, or of more pieces than a wavefront has lanes: a pair of pieces to a lane, what is left element by element.
template <typename T>
__global__ void __launch_bounds__(256) k_cache_append(AppendArgs a, AppendUnits n)
{
    constexpr int VE = 16 / sizeof(T), ES = sizeof(T);
    __shared__ AppendShared sh;
    const int tid = threadIdx.x;
    const int64_t token0 = (int64_t)blockIdx.x * n.per;
    const int count = (int)std::min<int64_t>(n.per, a.tokens - token0);
    const CacheView &c = a.c;
    const int d = c.head_dim, pairs = a.rotary / 2;
    append_places(a, token0, count, sh);
    const auto &turn = sh.turn;
    const auto &at = sh.at;
    const int group = n.groups > 1 ? tid / n.all : 0;
    if (group >= n.groups)
        return;
    for (int u = n.groups > 1 ? tid - group * n.all : blockIdx.y * 256 + tid; u < n.all; u += 256 * gridDim.y) {
        // the unit: where its one or two pieces come from and go to in a token.  All pairs of pieces, then what is copied: a wavefront is
        // mostly of one kind.
        const char *from;
        char *to;
        int64_t from_token, to_token = -1;
        const bool turns = u < n.turning;
        const int r = turns ? u / n.n_pair : (u - n.turning) / n.n_rest, w = turns ? u - r * n.n_pair : (u - n.turning) - r * n.n_rest;
        int at_a, at_b, j = 0, left = VE;  // bytes in the row; first pair; pairs or elements there
        if (!turns && u >= n.turning + n.resting) {
            const int h = (u - n.turning - n.resting) / n.n_v;
            at_a = at_b = piece_start((u - n.turning - n.resting) - h * n.n_v, d * ES);
            from = a.v + h * a.v_head, from_token = a.v_token;
            to = c.v + h * c.head_stride;
        } else {
            if (r < a.q_heads) {
                from = a.q + r * a.q_head, from_token = a.q_token;
                to = a.qo + r * a.qo_head, to_token = a.qo_token;
            } else {
                from = a.k + (r - a.q_heads) * a.k_head, from_token = a.k_token;
                to = c.k + (r - a.q_heads) * c.head_stride;
            }
            if (turns) {
                j = w * VE, left = pairs - j;
                // fewer pairs than a piece has: the row's last ones (some are then turned twice, which a row in place does not bear)
                if (left < VE && pairs >= VE && !(n.in_place && r < a.q_heads))
                    j = pairs - VE, left = VE;
                at_a = (a.interleaved ? 2 * j : j) * ES, at_b = a.interleaved ? at_a + 16 : (pairs + j) * ES;
            } else {
                const int e = a.rotary + w * VE;
                left = d - e;
                at_a = at_b = left < VE && d - VE >= a.rotary ? (d - VE) * ES : e * ES;
                if (at_a != e * ES)
                    left = VE;
            }
        }
        auto target = [&](int t) { return to + (to_token < 0 ? at[t] : (token0 + t) * to_token); };
        auto source = [&](int t) { return from + (token0 + t) * from_token; };
        if (left >= VE) {
            for (int t0 = group; t0 < count; t0 += kAppendDeep * n.groups) {
                Piece16<T> x[kAppendDeep], y[kAppendDeep];
#pragma unroll
                for (int i = 0; i < kAppendDeep; ++i) {
                    const char *const p = source(std::min(t0 + i * n.groups, count - 1));
                    x[i] = *(const Piece16<T> *)(p + at_a);
                    if (turns)
                        y[i] = *(const Piece16<T> *)(p + at_b);
                }
#pragma unroll
                for (int i = 0; i < kAppendDeep; ++i) {
                    const int t = t0 + i * n.groups;
                    if (t >= count || at[t] < 0)
                        continue;
                    if (turns) {
                        const float *const cs = turn[t][0] + j, *const sn = turn[t][1] + j;
                        if (a.interleaved) {
#pragma unroll
                            for (int e = 0; e < VE / 2; ++e) {
                                rotate_pair(x[i].v[2 * e], x[i].v[2 * e + 1], cs[e], sn[e]);
                                rotate_pair(y[i].v[2 * e], y[i].v[2 * e + 1], cs[VE / 2 + e], sn[VE / 2 + e]);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < VE; ++e)
                                rotate_pair(x[i].v[e], y[i].v[e], cs[e], sn[e]);
                        }
                        *(Piece16<T> *)(target(t) + at_b) = y[i];
                    }
                    *(Piece16<T> *)(target(t) + at_a) = x[i];
                }
            }
        } else {  // element by element
            for (int t = group; t < count; t += n.groups) {
                if (at[t] < 0)
                    continue;
                const T *const f = (const T *)source(t);
                T *const o = (T *)target(t);
                if (!turns) {
                    for (int e = d - left; e < d; ++e)
                        o[e] = f[e];
                } else {
                    for (int e = j; e < pairs; ++e) {
                        const int p = a.interleaved ? 2 * e : e, q = a.interleaved ? 2 * e + 1 : pairs + e;
                        T x = f[p], y = f[q];
                        rotate_pair(x, y, turn[t][0][e], turn[t][1][e]);
                        o[p] = x, o[q] = y;
                    }
                }
            }
        }
    }
}

int check_append(const tig_cache *c, const tig_cache_append *p)
{
    int rc = check_cache(c);
    if (rc != TIG_OK)
        return rc;
    if (!p || p->struct_size != sizeof(tig_cache_append))
        return fail_text(TIG_EINVAL, "tig_cache_append: NULL argument or wrong struct_size");
    if ((rc = check_sequences(*c, p->seqs, p->table, p->ld_table, p->lengths)) != TIG_OK)
        return rc;
    if (p->rotary < 0 || p->rotary > c->head_dim || p->rotary % 2 || p->interleaved < 0 || p->interleaved > 1 || p->reserved != 0)
        return fail_text(TIG_EINVAL, "tig_cache_append: rotary or interleaved out of range, or reserved is not 0");
    if (p->tokens < 0 || p->tokens > (1 << 23) || (!p->starts && p->tokens != p->seqs))
        return fail_text(TIG_EINVAL, "tig_cache_append: tokens out of range, or not one for each sequence without starts");
    if (p->position_type < 0 || p->position_type > 2 || (p->tokens > 0 && (p->position_type != 0) != (p->positions != nullptr)) ||
        ((p->rotary > 0) != (p->freq != nullptr)) || !element_aligned(p->positions, 8) || !element_aligned(p->freq, 8) || !element_aligned(p->starts, 4))
        return fail_text(TIG_EINVAL, "tig_cache_append: positions do not go with position_type, or freq with rotary, or one is not aligned");
    if (p->q_heads < 0 || p->q_heads > (1 << 14) || (p->tokens > 0 && ((p->q_heads != 0) != (p->q != nullptr) || (p->q != nullptr) != (p->q_out != nullptr))))
        return fail_text(TIG_EINVAL, "tig_cache_append: q, q_out and q_heads do not go together, or q_heads is out of range");
    const int es = dtype_bytes(c->dtype);
    if (p->tokens > 0 && (!p->k || !p->v))
        return fail_text(TIG_EINVAL, "tig_cache_append: k or v is NULL");
    if (!element_aligned(p->k, es) || !element_aligned(p->v, es) || !element_aligned(p->q, es) || !element_aligned(p->q_out, es))
        return fail_text(TIG_EINVAL, "tig_cache_append: an address is not aligned to its element");
    for (const int64_t s : {p->k_token, p->k_head, p->v_token, p->v_head, p->q_token, p->q_head, p->qo_token, p->qo_head})
        if (s < 0 || s > ((int64_t)1 << 32))
            return fail_text(TIG_EINVAL, "tig_cache_append: a stride is out of range");
    if (p->q_out && rows_meet(p->tokens, p->qo_token, p->q_heads, p->qo_head, c->head_dim))
        return fail_text(TIG_EINVAL, "tig_cache_append: rows of q_out overlap");
    return TIG_OK;
}

int check_append_apart(const tig_cache &c, const tig_cache_append &p)
{
    const int es = dtype_bytes(c.dtype);
    const int64_t n = p.tokens;
    auto rows = [&](const void *x, int64_t token, int64_t heads, int64_t head) { return placed(x, {{n, token}, {heads, head}}, c.head_dim, es); };
    const bool in_place = p.q == p.q_out && p.q_token == p.qo_token && p.q_head == p.qo_head;
    const Placed in[] = {rows(p.k, p.k_token, c.heads, p.k_head), rows(p.v, p.v_token, c.heads, p.v_head), rows(in_place ? nullptr : p.q, p.q_token, p.q_heads, p.q_head),
                         {p.table, p.seqs, c.max_pages, p.ld_table, 4}, {p.lengths, 1, p.seqs, p.seqs, 4}, {p.starts, 1, p.seqs + 1, p.seqs + 1, 4},
                         {p.positions, 1, n, n, 8}, {p.freq, 1, p.rotary / 2, p.rotary / 2, 8}};
    const Placed out[] = {placed_keys(c, c.k), placed_keys(c, c.v), rows(p.q_out, p.qo_token, p.q_heads, p.qo_head)};
    return all_apart(in, out) ? TIG_OK : fail_text(TIG_EINVAL, "tig_cache_append: an output overlaps another tensor of the call");
}

// ------------------------------------------------------------------------------------------
// Sequences that are taken over: a workgroup's share of a last page's rows; the first of a sequence's also writes its table.  Bound by memory:
// 2048 sequences' pages of up to 63 rows of 4 x 256 bytes 51 us (262 MB, 5.1 TB/s), 16 of up to 15 rows of 8 x 256 bytes 3.9 us.

struct ForkArgs {
    CacheView c;
    int64_t rows_in, rows_out, ld_out;
    const int32_t *parents, *spare;
    int32_t *table_out, *lengths_out;
    int32_t heads_inner;  // heads lie closer together than rows
};

__global__ void __launch_bounds__(256) k_cache_fork(ForkArgs a, int es)
{
    const CacheView &c = a.c;
    const int64_t r = blockIdx.x;
    const int64_t parent = a.parents[r];
    const bool some = parent >= 0 && parent < a.rows_in;
    const int length = some ? c.length(parent) : 0;
    const int n = c.div.quotient(length), left = length - n * c.page_size;
    const int32_t *const from = c.table + (some ? parent : 0) * c.ld_table;
    const int spare = a.spare[r], last = left > 0 ? from[n] : -1;
    const bool copies = left > 0 && c.page_ok(spare) && c.page_ok(last);
    if (blockIdx.y == 0) {
        for (int i = threadIdx.x; i < c.max_pages; i += 256)
            a.table_out[r * a.ld_out + i] = i < n ? from[i] : i > n ? -1 : left > 0 && !copies ? last : c.page_ok(spare) ? spare : -1;
        if (threadIdx.x == 0)
            a.lengths_out[r] = length;
    }
    if (!copies)
        return;
    const int row_bytes = c.head_dim * es, pieces = (row_bytes + 15) / 16, per_cache = left * c.heads * pieces;
    const int inner = a.heads_inner ? c.heads : left;
    for (int u = blockIdx.y * 256 + threadIdx.x; u < 2 * per_cache; u += 256 * gridDim.y) {
        char *const base = u < per_cache ? c.k : c.v;
        const int w = u < per_cache ? u : u - per_cache, x = w / pieces, o = x / inner, i = x % inner;
        const int row = a.heads_inner ? o : i, head = a.heads_inner ? i : o, at = piece_start(w % pieces, row_bytes);
        *(Sixteen *)(base + c.offset(spare, row, head) + at) = *(const Sixteen *)(base + c.offset(last, row, head) + at);
    }
}

int check_fork(const tig_cache *c, const tig_cache_fork *p)
{
    int rc = check_cache(c);
    if (rc != TIG_OK)
        return rc;
    if (!p || p->struct_size != sizeof(tig_cache_fork) || p->reserved != 0)
        return fail_text(TIG_EINVAL, "tig_cache_fork: NULL argument, wrong struct_size, or reserved is not 0");
    if (p->rows_out < 0 || p->rows_out > (1 << 20))
        return fail_text(TIG_EINVAL, "tig_cache_fork: rows_out out of range");
    if ((rc = check_sequences(*c, p->rows_in, p->table, p->ld_table, p->lengths)) != TIG_OK)
        return rc;
    if (p->rows_out > 0 && (!p->parents || !p->spare || !p->table_out || !p->lengths_out))
        return fail_text(TIG_EINVAL, "tig_cache_fork: parents, spare, table_out or lengths_out is NULL");
    if (!element_aligned(p->parents, 4) || !element_aligned(p->spare, 4) || !element_aligned(p->table_out, 4) || !element_aligned(p->lengths_out, 4))
        return fail_text(TIG_EINVAL, "tig_cache_fork: an address is not aligned to its element");
    if (p->ld_out < c->max_pages || p->ld_out > ((int64_t)1 << 32))
        return fail_text(TIG_EINVAL, "tig_cache_fork: the table's row stride is smaller than max_pages or above 2^32");
    const Placed in[] = {{p->table, p->rows_in, c->max_pages, p->ld_table, 4}, {p->lengths, 1, p->rows_in, p->rows_in, 4},
                         {p->parents, 1, p->rows_out, p->rows_out, 4}, {p->spare, 1, p->rows_out, p->rows_out, 4}};
    const Placed out[] = {{p->table_out, p->rows_out, c->max_pages, p->ld_out, 4}, {p->lengths_out, 1, p->rows_out, p->rows_out, 4}, placed_keys(*c, c->k),
                          placed_keys(*c, c->v)};
    return all_apart(in, out) ? TIG_OK : fail_text(TIG_EINVAL, "tig_cache_fork: an output overlaps another tensor of the call");
}

}  // namespace

}  // namespace tig

using namespace tig;

int tig_cache_append_run(const tig_cache *cache, const tig_cache_append *p, void *hip_stream)
{
    int rc = check_append(cache, p);
    if (rc != TIG_OK || p->tokens == 0 || p->seqs == 0)
        return rc;
    if ((rc = check_append_apart(*cache, *p)) != TIG_OK)
        return rc;
    const int64_t es = dtype_bytes(cache->dtype);
    AppendArgs a = {};
    a.c = cache_view(*cache, p->table, p->ld_table, p->lengths);
    a.seqs = p->seqs, a.tokens = p->tokens, a.starts = p->starts, a.positions = p->positions, a.freq = p->freq;
    a.k = (const char *)p->k, a.v = (const char *)p->v, a.q = (const char *)p->q, a.qo = (char *)p->q_out;
    a.k_token = p->k_token * es, a.k_head = p->k_head * es, a.v_token = p->v_token * es, a.v_head = p->v_head * es;
    a.q_token = p->q_token * es, a.q_head = p->q_head * es, a.qo_token = p->qo_token * es, a.qo_head = p->qo_head * es;
    a.q_heads = p->q_heads, a.rotary = p->rotary, a.interleaved = p->interleaved, a.position_type = p->position_type;
    const int ve = (int)(16 / es), d = cache->head_dim;
    AppendUnits n = {};
    n.in_place = p->q != nullptr && p->q == p->q_out;
    const int part = p->interleaved ? p->rotary : p->rotary / 2, rest = d - p->rotary;
    const int in_part = (part + ve - 1) / ve, in_row = std::max((p->interleaved ? 1 : 2) * in_part + (rest + ve - 1) / ve, (d + ve - 1) / ve);
    const bool pieces = (part == 0 || part >= ve) && (rest == 0 || rest >= ve) && in_row <= 64;  // parts of a piece at least, a row in a wavefront
    if (pieces) {
        n.n_pair = in_part;
        while (1 << n.shift < in_row)
            ++n.shift;
        n.all = (p->q_heads + 2 * cache->heads) << n.shift;
    } else {
        n.n_pair = (p->rotary / 2 + ve - 1) / ve;
        n.n_rest = std::max(1, (d - p->rotary + ve - 1) / ve);  // (a divisor)
        n.n_v = (d + ve - 1) / ve;
        n.turning = (p->q_heads + cache->heads) * n.n_pair;
        n.resting = p->rotary < d ? (p->q_heads + cache->heads) * n.n_rest : 0;
        n.all = n.turning + n.resting + cache->heads * n.n_v;
        n.groups = std::max(1, 256 / n.all);
    }
    // a workgroup's tokens: as many as leave about four workgroups for a compute unit
    n.per = (int)std::min<int64_t>(kAppendTokens, std::max<int64_t>(1, p->tokens / 1024));
    // ... and a few tokens' rows by several workgroups (one token of 48 rows of 256 bytes: 5.0 us by one, 3.5 by three)
    const int64_t groups = (p->tokens + n.per - 1) / n.per, shares = groups <= 256 ? (n.all + 255) / 256 : 1;
    const dim3 grid((unsigned)groups, (unsigned)shares);
    with_dtype(cache->dtype, [&](auto t) {
        using T = decltype(t);
        auto *const rows = n.in_place ? k_cache_append_rows<T, true> : k_cache_append_rows<T, false>;
        hipLaunchKernelGGL((pieces ? rows : k_cache_append<T>), grid, dim3(256), 0, (hipStream_t)hip_stream, a, n);
        return 0;
    });
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TIG_OK : fail_global("tig_cache_append_run", e);
}

int tig_cache_fork_run(const tig_cache *cache, const tig_cache_fork *p, void *hip_stream)
{
    const int rc = check_fork(cache, p);
    if (rc != TIG_OK || p->rows_out == 0)
        return rc;
    const int es = dtype_bytes(cache->dtype);
    ForkArgs a = {};
    a.c = cache_view(*cache, p->table, p->ld_table, p->lengths);
    a.rows_in = p->rows_in, a.rows_out = p->rows_out, a.ld_out = p->ld_out;
    a.parents = p->parents, a.spare = p->spare, a.table_out = p->table_out, a.lengths_out = p->lengths_out;
    a.heads_inner = cache->head_stride <= cache->token_stride;
    const int64_t pieces = 2 * (int64_t)cache->page_size * cache->heads * ((cache->head_dim * es + 15) / 16);
    const int64_t blocks = std::min<int64_t>(std::max<int64_t>(1, pieces / 2048), 64);
    hipLaunchKernelGGL(k_cache_fork, dim3((unsigned)p->rows_out, (unsigned)blocks), dim3(256), 0, (hipStream_t)hip_stream, a, es);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TIG_OK : fail_global("tig_cache_fork_run", e);
}
