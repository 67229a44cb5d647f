// The k best continuations over beams and vocabulary (include/tig.h, tig_beam_select).  gfx950.
//
//   score of candidate (j, v) = scores_j + l_jv - log sum_u exp l_ju, the k largest, ties to the lowest (j, v)
//
//   k_select_segments  reads the logits once: for every segment (`group` times 128 logits, 512 apart) its largest logit, for every
//                      wavefront's stretch the sum of exp(l - largest); bound by memory
//   k_select_pick      a workgroup per batch entry: log-sums from the segments'; a bound that at least k candidates reach; the few
//                      segments that reach it are read again, and the candidates at or above it are ranked
// Which bound: the segments are dealt in turn to 128 groups, and the k-th largest of the groups' maxima is the score of a candidate that
// k - 1 others reach at least.  For values in no particular order, also where one beam has all the best, a few more than k lie above it;
// whatever order they are in, nothing above it is missed.  Where more than 128 candidates reach it, the candidates themselves are dealt to the
// groups for a better one.  Scores are compared in fp64: candidates of one beam in the order of their logits, those of several beams, and
// finished ones beside them, with log-sums of fp32 exponentials.  These are off by 1e-8 where many logits carry the sum (a million of standard deviation 1:
// 5e-9), by 1.4e-7 where one distance does (a peak over equal logits: an argument's rounding and the function's own are then all alike), by
// 64 units of 2^-24 at most where beams * vocab is up to 2^23: 27 roundings on the way of a sum, two of an argument, which is ln vocab on average at
// most, and the function's two.  (Rows beyond that have longer stretches: five more roundings for every four steps of 512 logits.)
//
// 50 x 8 rows of 250,000 in bf16, k = 8: 46 us (37 the logits, 200 MB at 5.4 TB/s); 129 rows of 1,000,003 in fp32, k = 100: 113 us (93, 516 MB at
// 5.6 TB/s); 4 rows of 32,000, k = 4: 12 us, two launches of a chain of round trips each.
#include <cmath>

#include "cache.h"

namespace tig {

namespace {

struct SelectArgs {
    const void *logits;
    int64_t l_batch, l_beam;  // elements
    int64_t batch;
    int32_t beams, k, vocab;
    // A row: `blocks` steps of 512 logits, each sixteen lanes' 128 of them; segments of `group` steps, 4 each; a wavefront's stretch is `per`
    // steps (whole groups).
    int32_t blocks, group, per, stretches, segments;
    PageDiv by_segments, by_eights;  // divisions by a row's segments, and by the eights of a segment
    const float *scores;
    const uint8_t *finished;
    int32_t end;
    float *top;     // [batch x beams][segments]: largest logit of segment 4 (step / group) + (lane / 16)
    float2 *sums;   // [batch x beams][stretches]: largest logit, sum of exp(l - largest)
    float *scores_out;
    int32_t *parents, *tokens;
    uint8_t *finished_out;
};

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight {
    T v[8];
};

// logits at .. at + 7 of a row; -infinity behind its end
template <typename T>
__device__ inline void load_eight(const T *row, int at, int vocab, float (&x)[8])
{
    if (at + 8 <= vocab) {
        const Eight<T> q = *(const Eight<T> *)(row + at);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = to_float(q.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = at + e < vocab ? to_float(row[at + e]) : -INFINITY;
    }
}

// exp(x), x <= 0.  log2 e in two parts: in fp32 alone it is 1.3e-8 of itself short, which makes every exponential that much of its argument too large,
// always to one side, and a sum of however many keeps it (2.5e-8 of a million logits of standard deviation 1; 35.2 us for 200 MB of bf16 with one part,
// 37 with both).
constexpr float kLog2e = 1.44269504f, kLog2eRest = 1.92596299e-8f;
__device__ inline float exp_below(float x) { return __builtin_amdgcn_exp2f(fmaf(x, kLog2e, x * kLog2eRest)); }

// written out: the compiler would canonicalise every operand.  A NaN loses: the row's sum has it.
__device__ inline float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// the maxima of four values over each sixteen lanes (four at once: a read of a register just written would have to wait)
__device__ inline void row_max_four(float (&v)[4])
{
    asm volatile("s_nop 1\n\t"
                 "v_max_f32_dpp %0, %0, %0 row_ror:1 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %1, %1, %1 row_ror:1 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %2, %2, %2 row_ror:1 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %3, %3, %3 row_ror:1 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %0, %0, %0 row_ror:2 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %1, %1, %1 row_ror:2 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %2, %2, %2 row_ror:2 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %3, %3, %3 row_ror:2 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %0, %0, %0 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %1, %1, %1 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %2, %2, %2 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %3, %3, %3 row_ror:4 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %1, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %2, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
                 "v_max_f32_dpp %3, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
                 "s_nop 1"
                 : "+v"(v[0]), "+v"(v[1]), "+v"(v[2]), "+v"(v[3]));
}

template <typename T>
__global__ void __launch_bounds__(256) k_select_segments(SelectArgs a)
{
    constexpr int kDeep = 4;  // steps whose logits are on their way together
    const int lane = lane_id();
    const int64_t id = (int64_t)blockIdx.x * 4 + wave_id_uniform();
    const int64_t r = id / a.stretches;
    const int stretch = (int)(id - r * a.stretches);
    if (r >= a.batch * a.beams)
        return;
    const bool done = a.finished && a.finished[r];
    float m = -INFINITY, s = 0.0f, seg = -INFINITY;
    const T *const row = (const T *)a.logits + r / a.beams * a.l_batch + r % a.beams * a.l_beam;
    const int s0 = stretch * a.per, s1 = std::min(a.blocks, s0 + a.per);
    int place = 0, within = 0;  // the segment of the sixteen that are collected, a lane each, and the step in it
    int first = s0 / a.group;   // the first of them
    auto flush = [&]() {
        const int n = (first + lane % 16) * 4 + lane / 16;
        if (lane % 16 < place && n < a.segments)
            a.top[r * a.segments + n] = seg;
        first += 16, place = 0, seg = -INFINITY;
    };
    auto add = [&](int t0, const float (&x)[kDeep][8]) {
        float top4[kDeep], top = m;
#pragma unroll
        for (int t = 0; t < kDeep; ++t) {
            top4[t] = max3(x[t][0], x[t][1], x[t][2]);
            top4[t] = max3(x[t][3], x[t][4], top4[t]);
            top4[t] = max3(x[t][5], x[t][6], top4[t]);
            top4[t] = max3(x[t][7], top4[t], top4[t]);
            top = fmaxf(top, top4[t]);
        }
        const float from = top == -INFINITY ? 0.0f : top;
        float sums[kDeep];
#pragma unroll
        for (int t = 0; t < kDeep; ++t) {
            sums[t] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sums[t] += exp_below(x[t][e] - from);
        }
        s *= exp_below(m - from);
#pragma unroll
        for (int t = 0; t < kDeep; ++t)
            s += sums[t];
        m = top;
        row_max_four(top4);
#pragma unroll
        for (int t = 0; t < kDeep; ++t) {
            if (t0 + t >= s1)
                break;
            seg = lane % 16 == place ? fmaxf(seg, top4[t]) : seg;
            if (++within == a.group) {
                within = 0;
                if (++place == 16)
                    flush();
            }
        }
    };
    int t0 = s0;
    if (!done)
        for (; t0 + kDeep <= s1 && (t0 + kDeep) * 512 <= a.vocab; t0 += kDeep) {
            float x[kDeep][8];
            Eight<T> q[kDeep];
#pragma unroll
            for (int t = 0; t < kDeep; ++t)
                q[t] = *(const Eight<T> *)(row + (t0 + t) * 512 + lane * 8);
#pragma unroll
            for (int t = 0; t < kDeep; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[t][e] = to_float(q[t].v[e]);
            add(t0, x);
        }
    for (; t0 < s1; t0 += kDeep) {
        float x[kDeep][8];
#pragma unroll
        for (int t = 0; t < kDeep; ++t)
            if (!done && t0 + t < s1) {
                load_eight(row, (t0 + t) * 512 + lane * 8, a.vocab, x[t]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[t][e] = -INFINITY;
            }
        add(t0, x);
    }
    if (within > 0)
        ++place;
    if (place > 0)
        flush();
    const float top = wave_max_all(m);
    s = wave_sum_all(s * exp_below(m - (top == -INFINITY ? 0.0f : top)));
    if (lane == 0)
        a.sums[r * a.stretches + stretch] = {top, s};
}

constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64, kGroups = 128, kMaxBeams = 64, kMaxK = 128;
constexpr int kMaxSegments = 8192;  // of a batch entry
constexpr int kRoom = 2048;         // candidates in LDS

struct PickShared {
    double top[kMaxBeams], log_sum[kMaxBeams], score[kMaxBeams];  // a row's log-sum-exp is top + log_sum: beside a mask of -3e38 one number loses the sum
    double part_sum[kPickWaves];
    float part_max[kPickWaves];
    double tops[kPickThreads], group[kGroups];
    double bound;
    int count, listed;
    int is_finished[kMaxBeams];
    alignas(16) double value[kRoom];
    int32_t id[kRoom];
    int32_t list[kMaxSegments];
};

// descending by value, then ascending by id
__device__ inline bool before(double va, int32_t ia, double vb, int32_t ib) { return va > vb || (va == vb && ia < ib); }

// puts the first `n` candidates into their order
__device__ inline void sort_candidates(PickShared &sh, int n)
{
    int size = 64;
    while (size < n)
        size *= 2;
    for (int i = n + threadIdx.x; i < size; i += kPickThreads)
        sh.value[i] = -INFINITY, sh.id[i] = 0x7fffffff;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            const int i = threadIdx.x / j * 2 * j + threadIdx.x % j, o = i + j;
            if (o < size) {
                const double vi = sh.value[i], vo = sh.value[o];
                const int32_t ii = sh.id[i], io = sh.id[o];
                if (before(vo, io, vi, ii) == ((i & k) == 0))
                    sh.value[i] = vo, sh.value[o] = vi, sh.id[i] = io, sh.id[o] = ii;
            }
            __syncthreads();
        }
}

// the k-th largest of the groups' maxima, of every thread's `top`
__device__ inline double group_bound(PickShared &sh, double top, int k)
{
    constexpr int kParts = kPickThreads / kGroups;
    const int tid = threadIdx.x, t = tid / kParts, part = tid % kParts;
    sh.tops[tid] = top;
    __syncthreads();
    if (tid < kGroups) {
#pragma unroll
        for (int i = 1; i < kParts; ++i)
            top = fmax(top, sh.tops[tid + i * kGroups]);
        sh.group[tid] = top;
    }
    __syncthreads();
    const double mine = sh.group[t];
    int rank = 0;
#pragma unroll
    for (int i = 0; i < kGroups; i += kParts)
        rank += before(sh.group[i + part], i + part, mine, t);
#pragma unroll
    for (int d = 1; d < kParts; d *= 2)
        rank += __shfl_xor(rank, d);
    if (part == 0 && rank == k - 1)
        sh.bound = mine;
    __syncthreads();
    return sh.bound;
}

// drops candidates below a better bound, if that is one
__device__ inline double raise_bound(PickShared &sh, double bound, int k)
{
    static_assert(kRoom == 2 * kPickThreads, "");
    const int tid = threadIdx.x, n = sh.count;
    double v[2];
    int32_t id[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int at = tid + i * kPickThreads;
        v[i] = at < n ? sh.value[at] : -INFINITY, id[i] = at < n ? sh.id[at] : 0;
    }
    const double better = group_bound(sh, fmax(v[0], v[1]), k);
    if (better <= bound)
        return bound;
    if (tid == 0)
        sh.count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (tid + i * kPickThreads < n && v[i] >= better) {
            const int at = atomicAdd(&sh.count, 1);
            sh.value[at] = v[i], sh.id[at] = id[i];
        }
    __syncthreads();
    return better;
}

template <typename T>
__global__ void __launch_bounds__(kPickThreads) k_select_pick(SelectArgs a)
{
    __shared__ PickShared sh;
    const int tid = threadIdx.x, lane = lane_id(), wave = wave_id_uniform();
    const int64_t b = blockIdx.x;
    const int per_beam = a.segments, all = a.beams * per_beam, n_sums = a.stretches;
    const float *const seg = a.top + b * all;
    const float2 *const sums = a.sums + b * a.beams * n_sums;
    constexpr int kMine = kMaxSegments / kPickThreads;
    float mine[kMine];  // the thread's segments tid, tid + 1024, ..: asked for ahead of all else
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        mine[i] = seg[std::min(tid + i * kPickThreads, all - 1)];
    // log-sums: some wavefronts per beam
    const int per = std::min(std::max(1, kPickWaves / a.beams), (n_sums + 63) / 64);  // wavefronts of a beam: a sum or two for each lane
    for (int j0 = 0; j0 < a.beams; j0 += kPickWaves / per) {
        const int j = j0 + wave / per, part = wave % per;
        const bool is = j < a.beams && wave / per < kPickWaves / per;
        float m = -INFINITY;
        if (is)
            for (int i = part * 64 + lane; i < n_sums; i += per * 64)
                m = fmaxf(m, sums[j * n_sums + i].x);
        m = wave_max_all(m);
        double s = 0.0;
        if (is)
            for (int i = part * 64 + lane; i < n_sums; i += per * 64) {
                const float2 x = sums[j * n_sums + i];
                s += x.x == -INFINITY ? (double)x.y : (double)x.y * exp((double)x.x - (double)m);
            }
#pragma unroll
        for (int d = 1; d < 64; d *= 2)
            s += __shfl_xor(s, d);
        if (lane == 0)
            sh.part_max[wave] = m, sh.part_sum[wave] = s;
        __syncthreads();
        if (tid < kPickWaves / per && j0 + tid < a.beams) {
            float top = -INFINITY;
            for (int i = 0; i < per; ++i)
                top = fmaxf(top, sh.part_max[tid * per + i]);
            double sum = 0.0;
            for (int i = 0; i < per; ++i) {
                const float o = sh.part_max[tid * per + i];
                sum += o == -INFINITY ? sh.part_sum[tid * per + i] : sh.part_sum[tid * per + i] * exp((double)o - (double)top);
            }
            const int64_t row = b * a.beams + j0 + tid;
            sh.top[j0 + tid] = (double)top, sh.log_sum[j0 + tid] = log(sum);
            sh.score[j0 + tid] = a.scores ? (double)a.scores[row] : 0.0;
            sh.is_finished[j0 + tid] = a.finished && a.finished[row];
        }
        __syncthreads();
    }
    auto value = [&](float logit, int j) {
        const double v = (((double)logit - sh.top[j]) - sh.log_sum[j]) + sh.score[j];
        return v > -INFINITY && logit > -INFINITY ? v : (double)-INFINITY;  // (NaN is none)
    };
    // the bound
    double here[kMine], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int n = tid + i * kPickThreads;
        here[i] = -INFINITY;
        if (n < all) {
            const int j = a.by_segments.quotient(n);
            here[i] = sh.is_finished[j] ? (double)-INFINITY : value(mine[i], j);
        }
        top = fmax(top, here[i]);
    }
    if (tid == 0)
        sh.count = sh.listed = 0;
    double bound = group_bound(sh, top, a.k);
    auto push = [&](double v, int32_t id) {
        const int at = atomicAdd(&sh.count, 1);
        if (at < kRoom)
            sh.value[at] = v, sh.id[at] = id;
    };
    auto push_finished = [&]() {
        if (tid < a.beams && sh.is_finished[tid] && sh.score[tid] >= bound && sh.score[tid] > -INFINITY)
            push(sh.score[tid], tid * a.vocab + a.end);
    };
#pragma unroll
    for (int i = 0; i < kMine; ++i)
        if (here[i] >= bound && here[i] > -INFINITY)
            sh.list[atomicAdd(&sh.listed, 1)] = tid + i * kPickThreads;
    push_finished();
    __syncthreads();
    const int listed = sh.listed;
    // the i-th eight logits of the listed segments: their row, the first one's place there, the beam
    struct Place {
        const T *row;
        int at, j;
    };
    const int per_segment = a.group * 16;
    auto place = [&](int i) {
        const int of = a.by_eights.quotient(i), e = i - of * per_segment, n = sh.list[of], j = a.by_segments.quotient(n), c = n - j * per_beam;
        return Place{(const T *)a.logits + b * a.l_batch + j * a.l_beam, (c / 4 * a.group + e / 16) * 512 + c % 4 * 128 + e % 16 * 8, j};
    };
    const int eights = listed * per_segment;
    constexpr int kDeep = 4;
    for (int i0 = tid; i0 < eights; i0 += kDeep * kPickThreads) {
        Place p[kDeep];
        Eight<T> q[kDeep];
#pragma unroll
        for (int t = 0; t < kDeep; ++t) {
            p[t] = place(std::min(i0 + t * kPickThreads, eights - 1));
            if (a.vocab >= 8)  // (eight from the row's end where there are fewer left)
                q[t] = *(const Eight<T> *)(p[t].row + std::min(p[t].at, a.vocab - 8));
        }
#pragma unroll
        for (int t = 0; t < kDeep; ++t) {
            if (i0 + t * kPickThreads >= eights || p[t].at >= a.vocab)
                continue;
            const int first = a.vocab >= 8 ? std::min(p[t].at, a.vocab - 8) : 0, j = p[t].j;
            // the logit that reaches the bound, less a few roundings of it and of the score: whoever reaches that is looked at in fp64
            const float near = (float)(((bound - sh.score[j]) + sh.log_sum[j]) + sh.top[j]);
            const float size = (float)(fabs(bound) + fabs(sh.score[j]) + fabs(sh.log_sum[j]) + fabs(sh.top[j]));
            const float least = near - (fabsf(near) * 1e-6f + size * 1e-14f + 1e-30f);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = a.vocab >= 8 ? to_float(q[t].v[e]) : first + e < a.vocab ? to_float(p[t].row[e]) : -INFINITY;
                if (x < least || first + e < p[t].at || first + e >= a.vocab)
                    continue;
                const double v = value(x, j);
                if (v >= bound && v > -INFINITY)
                    push(v, j * a.vocab + first + e);
            }
        }
    }
    __syncthreads();
    if (sh.count > kRoom) {  // many of one value, or in an unlucky order: again, a thousand at a time, the k best of them kept
        __syncthreads();
        if (tid == 0)
            sh.count = 0;
        __syncthreads();
        push_finished();
        __syncthreads();
        int32_t bound_id = 0x7fffffff;  // of candidates at the bound, the last id that still counts
        for (int i0 = 0; i0 < eights; i0 += kPickThreads)
            for (int e = 0; e < 8; ++e) {
                if (sh.count > kRoom - kPickThreads) {
                    const double better = raise_bound(sh, bound, a.k);
                    if (better > bound)
                        bound = better, bound_id = 0x7fffffff;
                }
                __syncthreads();
                if (sh.count > kRoom - kPickThreads) {
                    const int n = sh.count;
                    sort_candidates(sh, n);
                    if (n >= a.k)
                        bound = sh.value[a.k - 1], bound_id = sh.id[a.k - 1];
                    if (tid == 0)
                        sh.count = n < a.k ? n : a.k;
                }
                __syncthreads();
                const int i = i0 + tid;
                if (i < eights) {
                    const Place p = place(i);
                    if (p.at + e < a.vocab) {
                        const double v = value(to_float(p.row[p.at + e]), p.j);
                        const int32_t id = p.j * a.vocab + p.at + e;
                        if ((v > bound || (v == bound && id <= bound_id)) && v > -INFINITY)
                            push(v, id);
                    }
                }
                __syncthreads();
            }
    }
    // (ranks cost the candidates' number squared: 10 x 4 rows of 303, k = 12, 15 us with a better bound for more than 128 of them, 29 for more than 512)
    if (sh.count > 128)
        bound = raise_bound(sh, bound, a.k);
    const int count = sh.count;
    auto write = [&](int rank, double v, int32_t id) {
        const int64_t o = b * a.k + rank;
        const int j = id < 0 ? 0 : id / a.vocab, token = id < 0 ? -1 : id - j * a.vocab;
        a.scores_out[o] = (float)v;
        a.parents[o] = id < 0 ? -1 : (int32_t)(b * a.beams + j);
        a.tokens[o] = token;
        if (a.finished_out)
            a.finished_out[o] = id >= 0 && (sh.is_finished[j] || token == a.end);
    };
    if (count <= 512) {  // each candidate's rank: how many come before it
        int parts = kPickThreads / 64;
        while (parts > 1 && kPickThreads / parts < count)
            parts /= 2;
        const int t = tid / parts, part = tid % parts;
        int rank = 0;
        if (t < count) {  // (the ids only where values are equal)
            const double v = sh.value[t];
            const int32_t id = sh.id[t];
            const int each = ((count + parts - 1) / parts + 1) / 2 * 2, end = std::min(count, (part + 1) * each);
#pragma unroll 4
            for (int i = part * each; i < end; i += 2) {
                const double2 o = *(const double2 *)&sh.value[i];
                rank += (o.x > v) + (i + 1 < end && o.y > v);
                if (o.x == v && i != t)
                    rank += sh.id[i] < id;
                if (o.y == v && i + 1 < end && i + 1 != t)
                    rank += sh.id[i + 1] < id;
            }
        }
        for (int d = 1; d < parts; d *= 2)
            rank += __shfl_xor(rank, d);
        if (t < count && part == 0 && rank < a.k)
            write(rank, sh.value[t], sh.id[t]);
    } else {
        sort_candidates(sh, count);
        if (tid < a.k && tid < count)
            write(tid, sh.value[tid], sh.id[tid]);
    }
    if (tid >= count && tid < a.k)
        write(tid, -INFINITY, -1);
}

struct SelectPlan {
    int blocks, group, per, stretches, segments;
    size_t sums, bytes;
};
// Segments as short as an entry's fit; stretches of up to 8 steps where there are wavefronts enough (129 rows of a million in fp32: 112 us, 112 with 16,
// 118 with 64; 400 rows of 250,000 in bf16: 59, 59, 65).
SelectPlan select_plan(const tig_beam_select &p)
{
    SelectPlan L = {};
    const int64_t blocks = (p.vocab + 511) / 512, rows = p.batch * p.beams;
    int64_t group = 1;
    while (p.beams * ((blocks + group - 1) / group) * 4 > kMaxSegments)
        ++group;
    int64_t per = std::min<int64_t>(8, std::max<int64_t>(1, rows * blocks / 8192));
    per = per > 4 ? 8 : per;
    while (rows * ((blocks + per - 1) / per) > (1 << 25))  // (a launch's threads fit 32 bits)
        per *= 2;
    per = (per + group - 1) / group * group;
    L.blocks = (int)blocks, L.group = (int)group, L.per = (int)per, L.stretches = (int)((blocks + per - 1) / per);
    L.segments = (int)((blocks + group - 1) / group * 4);
    L.sums = ((size_t)rows * L.segments * sizeof(float) + 255) / 256 * 256;
    L.bytes = (L.sums + (size_t)rows * L.stretches * sizeof(float2) + 255) / 256 * 256;
    return L;
}

int check_select(const tig_beam_select *p)
{
    if (!p || p->struct_size != sizeof(tig_beam_select))
        return fail_text(TIG_EINVAL, "tig_beam_select: NULL argument or wrong struct_size");
    if (!dtype_ok(p->dtype) || p->reserved != 0)
        return fail_text(TIG_EINVAL, "tig_beam_select: unknown dtype, or reserved is not 0");
    if (p->batch < 0 || p->batch > (1 << 20) || p->beams < 1 || p->beams > kMaxBeams || p->k < 1 || p->k > kMaxK || p->vocab < 1 || p->vocab > (1 << 28) ||
        p->beams * p->vocab > 0x7fffffff || p->batch * p->beams > (1 << 24))
        return fail_text(TIG_EINVAL, "tig_beam_select: batch, beams, k or vocab out of range");
    if (p->end < -1 || p->end >= p->vocab || (p->finished && p->end < 0))
        return fail_text(TIG_EINVAL, "tig_beam_select: end is no candidate (finished beams need one)");
    if (p->batch > 0 && (!p->logits || !p->scores_out || !p->parents || !p->tokens))
        return fail_text(TIG_EINVAL, "tig_beam_select: logits, scores_out, parents or tokens is NULL");
    const int64_t most = (int64_t)1 << 40;
    if (p->l_batch < 0 || p->l_beam < 0 || p->l_batch > most || p->l_beam > most)
        return fail_text(TIG_EINVAL, "tig_beam_select: a stride is out of range");
    if ((uintptr_t)p->logits % (uintptr_t)dtype_bytes(p->dtype) || (((uintptr_t)p->scores | (uintptr_t)p->scores_out | (uintptr_t)p->parents | (uintptr_t)p->tokens) & 3))
        return fail_text(TIG_EINVAL, "tig_beam_select: an address is not aligned to its element");
    return TIG_OK;
}

int check_select_apart(const tig_beam_select &p)
{
    const int64_t n = p.batch * p.beams, o = p.batch * p.k;
    const int es = dtype_bytes(p.dtype);
    // (what lies between the rows of logits counts as theirs)
    const int64_t span = (p.batch - 1) * p.l_batch + (p.beams - 1) * p.l_beam + p.vocab;
    const Placed in[] = {{p.logits, 1, span, span, es}, {p.scores, 1, n, n, 4}, {p.finished, 1, n, n, 1}};
    const Placed out[] = {{p.scores_out, 1, o, o, 4}, {p.parents, 1, o, o, 4}, {p.tokens, 1, o, o, 4}, {p.finished_out, 1, o, o, 1}};
    return all_apart(in, out) ? TIG_OK : fail_text(TIG_EINVAL, "tig_beam_select: an output overlaps another tensor of the call");
}

}  // namespace

}  // namespace tig

using namespace tig;

int tig_beam_select_workspace_bytes(const tig_beam_select *p, size_t *bytes)
{
    const int rc = check_select(p);
    if (rc != TIG_OK)
        return rc;
    if (!bytes)
        return fail_text(TIG_EINVAL, "tig_beam_select_workspace_bytes: bytes is NULL");
    *bytes = p->batch > 0 ? select_plan(*p).bytes : 0;
    return TIG_OK;
}

int tig_beam_select_run(const tig_beam_select *p, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_select(p);
    if (rc != TIG_OK || p->batch == 0)
        return rc;
    const SelectPlan L = select_plan(*p);
    if (!workspace || ((uintptr_t)workspace & 255))
        return fail_text(TIG_EINVAL, "tig_beam_select_run: workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < L.bytes)
        return fail_text(TIG_ENOSPACE, "tig_beam_select_run: workspace too small");
    if ((rc = check_select_apart(*p)) != TIG_OK)
        return rc;
    const hipStream_t s = (hipStream_t)hip_stream;
    SelectArgs a = {p->logits, p->l_batch, p->l_beam, p->batch, p->beams, p->k, (int32_t)p->vocab, L.blocks, L.group, L.per, L.stretches, L.segments, page_div(L.segments), page_div(L.group * 16),
                    p->scores, p->finished, p->end,
                    (float *)workspace, (float2 *)((char *)workspace + L.sums), p->scores_out, p->parents, p->tokens, p->finished_out};
    const int64_t waves = p->batch * p->beams * L.stretches;
    const hipError_t e = with_dtype(p->dtype, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((k_select_segments<T>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
        hipLaunchKernelGGL((k_select_pick<T>), dim3((unsigned)p->batch), dim3(kPickThreads), 0, s, a);
        return hipGetLastError();
    });
    return e == hipSuccess ? TIG_OK : fail_global("tig_beam_select_run", e);
}
