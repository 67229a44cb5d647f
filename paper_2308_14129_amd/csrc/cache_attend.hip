// Attention of single queries over sequences in a paged cache (include/tig.h, tig_cache_attend).  gfx950.
//
//   s_p = scale <q, k_p>,  out = sum_p exp(s_p - lse) v_p
//
// A unit is one sequence, one head of the cache and up to 16 QT of the query heads that share it; its rows go by in tiles of KT, one pass
// with a running maximum and sum.  The units' tiles stand in one long line (sequence by sequence, head by head), which is dealt evenly
// over all wavefronts: a wavefront works through its stretch of the line whatever sequences it crosses, so that one long sequence or
// four thousand short ones load the card alike.  What a wavefront has of a unit that it shares is joined with the other wavefronts' parts
// through LDS, and what a workgroup has of a unit that it shares through memory by a second launch, always in the line's order.
//
// Keys and values come straight from memory as operands of the matrix instructions, sixteen bytes a lane; nothing is staged:
//   scores       S[key][query] = K Q^T: a lane's sixteen bytes of a key row are its part of K's operand (lane % 16: the key), and
//                it ends with four keys of one query (lane % 16) in registers, which are the next product's operand as they are
//   values       O[column][query] = V^T P^T: V's operand wants several keys of one column; a lane loads adjacent columns
//                VE c .. (c = lane % 16) of the keys that it has the weights of, and one product takes the columns VE c + t of all c: packing the
//                t-th columns of two keys is one instruction
// Weights P are 16-bit operands in two parts, P = hi + lo: the matrix units have the time (a tile of 32 keys takes 16 KB through
// memory and less than half a microsecond of them), and one rounding of P would cost as much as rounding the output does.
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "cache.h"

namespace tig {

namespace {

struct AttendArgs {
    CacheView c;
    int64_t seqs;
    const char *q;
    char *out;
    float *lse;
    int64_t q_seq, q_head, o_seq, o_head;  // bytes
    int32_t q_heads, group, blocks, rows;  // query heads of a cache head, blocks of 16 QT of them, rows of a record
    int32_t window;
    uint32_t flip;                         // sign bits of Q, to keep the factor positive
    float scale, factor;                   // scale; |scale| log2(e)
    float *part;                           // [workgroups x 2] records: rows x (head_dim padded + 2)
    struct Tail *tails;                    // [workgroups]
    int64_t rec;                           // floats of a record
};
// The unit that a workgroup's stretch ends in, if it goes on in the next one's.
struct Tail {
    int32_t seq, unit, last;  // unit: head * blocks + block; last: the last workgroup that has a part of it, -1: none
};

constexpr int kAttendWaves = 4;

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <typename T>
struct AttendType;
template <>
struct AttendType<float> {
    static constexpr int KT = 16;
};
template <>
struct AttendType<__bf16> {
    static constexpr int KT = 32;
};
template <>
struct AttendType<_Float16> {
    static constexpr int KT = 32;
};

// rows [first, end) that sequence seq's query sees, and its tiles (one where it sees none, so that its output is written)
struct Seen {
    int first, end;
};
__device__ inline Seen seen(const CacheView &c, int window, int64_t seq)
{
    const int end = c.length(seq);
    return {window > 0 ? std::max(0, end - window) : 0, end};
}
template <int KT>
__device__ inline int tiles_of(const Seen &s)
{
    return std::max(1, (s.end + KT - 1) / KT - s.first / KT);
}

__device__ inline int64_t wave_sum_i64(int64_t v)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2)
        v += __shfl_xor(v, m);
    return v;
}

// maximum / sum over the four lanes that share lane % 16
__device__ inline float groups_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ inline float groups_sum(float v)
{
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// of a sum of weights; nothing was there: 0
__device__ inline float inverse(float total) { return total == 0.0f ? 0.0f : 1.0f / total; }
__device__ inline float log_sum(const AttendArgs &a, float top, float total) { return total == 0.0f ? -INFINITY : top * fabsf(a.scale) + logf(total); }

template <typename T, int DP, int QT, bool PAGED>
struct Attend {
    static constexpr int ES = sizeof(T), PE = 16 / ES, KT = AttendType<T>::KT, NS = KT / 16;
    static constexpr int NKB = DP / (4 * PE);             // blocks of k of the scores' product
    static constexpr int VE = ES == 2 && DP == 64 ? 4 : PE;  // columns of V that a lane loads at once
    static constexpr int NG = DP / (16 * VE);             // ... times
    static constexpr int VK = KT / 4;                     // keys of a lane
    // fp16 ends at 6e-8: a hundred thousand weights below that are not nothing beside one of 1
    static constexpr float kLift = std::is_same_v<T, _Float16> ? 16384.0f : 1.0f;

    struct Vpiece {
        int d[VE * ES / 4];
    };

    // per lane
    int lane, c16, g;
    int k_at[NKB];                 // byte of the lane's piece of a key row (and of q), -1: none
    int v_at[NG];
    int dup;                       // elements of the last block's piece that the one before has as well
    // per unit
    intx4 qv[QT][NKB];
    float m[QT], l[QT];
    floatx4 o[QT][NG * VE];

    __device__ inline void init(const AttendArgs &a)
    {
        lane = lane_id(), c16 = lane % 16, g = lane / 16;
        const int d = a.c.head_dim;
        dup = 0;
#pragma unroll
        for (int b = 0; b < NKB; ++b) {
            const int e = (b * 4 + g) * PE;
            k_at[b] = e >= d ? -1 : std::min(e, d - PE) * ES;
            if (e < d && e + PE > d)
                dup = e + PE - d;
        }
#pragma unroll
        for (int b = 0; b < NG; ++b) {
            const int e = (b * 16 + c16) * VE;
            v_at[b] = e >= d ? -1 : std::min(e, d - VE) * ES;
        }
    }
    // a piece's first `dup` elements are the piece before's: zero
    __device__ inline intx4 without_dup(intx4 x, int b, int d) const
    {
        if ((b * 4 + g) * PE + PE <= d)
            return x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (ES == 4) {
                if (i < dup)
                    x[i] = 0;
            } else {
                if (2 * i < dup)
                    x[i] &= 0xffff0000;
                if (2 * i + 1 < dup)
                    x[i] = 0;
            }
        }
        return x;
    }
    __device__ inline void begin(const AttendArgs &a, int64_t seq, int head, int block)
    {
        const int row0 = block * 16 * QT;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int row = row0 + 16 * t + c16;
            const bool is = row < a.group;
            const char *const p = a.q + seq * a.q_seq + (int64_t)(head * a.group + (is ? row : 0)) * a.q_head;
#pragma unroll
            for (int b = 0; b < NKB; ++b) {
                intx4 x = ((const Sixteen *)(p + std::max(k_at[b], 0)))->v;
                x = without_dup(x, b, a.c.head_dim);
                const uint32_t keep = is && k_at[b] >= 0 ? 0xffffffffu : 0u;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    qv[t][b][i] = (x[i] ^ a.flip) & keep;
            }
            m[t] = -INFINITY, l[t] = 0.0f;
#pragma unroll
            for (int i = 0; i < NG * VE; ++i)
                o[t][i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }

    // rows base .. base + KT - 1 of the sequence
    __device__ inline void tile(const AttendArgs &a, const int32_t *table, int head, int base, const Seen &s)
    {
        const CacheView &c = a.c;
        intx4 kv[NS][NKB];
        Vpiece vv[VK][NG];
        bool valid[VK];
        const int d = c.head_dim;
        if constexpr (PAGED) {  // sixteen rows lie in one page
            bool ok[NS];
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                const int at = base + 16 * t, n = c.div.quotient(at), r0 = at - n * c.page_size;
                const int page = at < s.end ? table[n] : -1;
                ok[t] = c.page_ok(page);
                const int64_t from = c.offset(ok[t] ? page : 0, r0, head);
                const int extent = ok[t] ? 15 * (int)c.token_stride + d * ES : 0;
                const auto kr = __builtin_amdgcn_make_buffer_rsrc((void *)(c.k + from), 0, extent, kBufferFlags);
                const auto vr = __builtin_amdgcn_make_buffer_rsrc((void *)(c.v + from), 0, extent, kBufferFlags);
                const int key = at + c16;
                const uint32_t row = key >= s.first && key < s.end ? (uint32_t)(c16 * (int)c.token_stride) : kBufferNone;
#pragma unroll
                for (int b = 0; b < NKB; ++b)
                    kv[t][b] = __builtin_bit_cast(intx4, __builtin_amdgcn_raw_buffer_load_b128(kr, (int)(k_at[b] < 0 ? kBufferNone : row + k_at[b]), 0, 0));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int vkey = at + 4 * g + i;
                    const bool in = vkey >= s.first && vkey < s.end;
                    valid[4 * t + i] = in && ok[t];
                    const uint32_t vrow = in ? (uint32_t)((4 * g + i) * (int)c.token_stride) : kBufferNone;
#pragma unroll
                    for (int b = 0; b < NG; ++b) {
                        const int off = (int)(v_at[b] < 0 ? kBufferNone : vrow + v_at[b]);
                        if constexpr (VE * ES == 16)
                            vv[4 * t + i][b] = __builtin_bit_cast(Vpiece, __builtin_amdgcn_raw_buffer_load_b128(vr, off, 0, 0));
                        else
                            vv[4 * t + i][b] = __builtin_bit_cast(Vpiece, __builtin_amdgcn_raw_buffer_load_b64(vr, off, 0, 0));
                    }
                }
            }
        } else {  // each row's page by itself; rows that are not there read another one's memory and count nothing
            int64_t from[NS];
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                const int key = base + 16 * t + c16;
                const bool in = key >= s.first && key < s.end;
                const int n = c.div.quotient(in ? key : 0);
                const int page = in ? table[n] : -1;
                from[t] = c.page_ok(page) ? c.offset(page, key - n * c.page_size, head) : -1;
                const char *const p = c.k + (from[t] < 0 ? head * c.head_stride : from[t]);
#pragma unroll
                for (int b = 0; b < NKB; ++b) {
                    kv[t][b] = ((const Sixteen *)(p + std::max(k_at[b], 0)))->v;
                    if (k_at[b] < 0)
                        kv[t][b] = intx4{0, 0, 0, 0};
                }
            }
#pragma unroll
            for (int t = 0; t < NS; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t f = __shfl(from[t], 4 * g + i);
                    valid[4 * t + i] = f >= 0;
                    const char *const p = c.v + (f < 0 ? head * c.head_stride : f);
                    struct __attribute__((packed, aligned(2))) Any {
                        Vpiece v;
                    };
#pragma unroll
                    for (int b = 0; b < NG; ++b) {
                        vv[4 * t + i][b] = ((const Any *)(p + std::max(v_at[b], 0)))->v;
#pragma unroll
                        for (int e = 0; e < VE * ES / 4; ++e)
                            vv[4 * t + i][b].d[e] = f < 0 ? 0 : vv[4 * t + i][b].d[e];
                    }
                }
        }
        if (d % PE != 0) {
#pragma unroll
            for (int t = 0; t < NS; ++t)
#pragma unroll
                for (int b = 0; b < NKB; ++b)
                    kv[t][b] = without_dup(kv[t][b], b, d);
        }
        // scores and weights
        float p[QT][VK];
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            float top = -INFINITY;
#pragma unroll
            for (int u = 0; u < NS; ++u) {
                floatx4 sc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int b = 0; b < NKB; ++b)
                    mma16(sc, kv[u][b], qv[t][b], T());
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[t][4 * u + i] = valid[4 * u + i] ? sc[i] : -INFINITY;
                    top = fmaxf(top, p[t][4 * u + i]);
                }
            }
            top = fmaxf(m[t], groups_max(top));
            const float from = top == -INFINITY ? 0.0f : top;
            const float keep = exp2_fast((m[t] - from) * a.factor);
            m[t] = top;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < VK; ++i) {
                p[t][i] = exp2_fast((p[t][i] - from) * a.factor);
                sum += p[t][i];
            }
            l[t] = l[t] * keep + sum;
#pragma unroll
            for (int i = 0; i < NG * VE; ++i)
                o[t][i] *= keep;
        }
        // values
        if constexpr (ES == 4) {
#pragma unroll
            for (int b = 0; b < NG; ++b)
#pragma unroll
                for (int e = 0; e < VE; ++e)
#pragma unroll
                    for (int t = 0; t < QT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            o[t][b * VE + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__int_as_float(vv[i][b].d[e]), p[t][i], o[t][b * VE + e], 0, 0, 0);
        } else {
            typedef T T8 __attribute__((ext_vector_type(8)));
            intx4 hi[QT], lo[QT];
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                T8 h, r;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float x = p[t][i] * kLift;
                    h[i] = (T)x;
                    r[i] = (T)(x - (float)h[i]);
                }
                hi[t] = __builtin_bit_cast(intx4, h), lo[t] = __builtin_bit_cast(intx4, r);
            }
#pragma unroll
            for (int b = 0; b < NG; ++b)
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    intx4 x;
#pragma unroll
                    for (int i = 0; i < 4; ++i)  // the e-th columns of keys 2 i and 2 i + 1
                        x[i] = (int)__builtin_amdgcn_perm((uint32_t)vv[2 * i + 1][b].d[e / 2], (uint32_t)vv[2 * i][b].d[e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                    for (int t = 0; t < QT; ++t) {
                        mma16(o[t][b * VE + e], x, lo[t], T());
                        mma16(o[t][b * VE + e], x, hi[t], T());
                    }
                }
        }
    }

    // the whole of a unit
    __device__ inline void finish(const AttendArgs &a, int64_t seq, int head, int block)
    {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float total = groups_sum(l[t]);
            const int row = block * 16 * QT + 16 * t + c16;
            if (row >= a.group)
                continue;
            const float by = inverse(total) * (1.0f / kLift);
            const int64_t q = (int64_t)head * a.group + row;
            if (a.lse && g == 0)
                a.lse[seq * a.q_heads + q] = log_sum(a, m[t], total);
            T *const out = (T *)(a.out + seq * a.o_seq + q * a.o_head);
            struct __attribute__((packed, aligned(sizeof(T)))) Out {
                T v[VE];
            };
#pragma unroll
            for (int b = 0; b < NG; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e0 = (b * 16 + 4 * g + i) * VE;
                    if (e0 < a.c.head_dim) {
                        Out x;
#pragma unroll
                        for (int e = 0; e < VE; ++e)
                            x.v[e] = (T)(o[t][b * VE + e][i] * by);
                        *(Out *)(out + std::min(e0, a.c.head_dim - VE)) = x;
                    }
                }
        }
    }
    // a part of a unit: `rows` rows of sums, then their maxima and the weights' sums
    __device__ inline void leave(const AttendArgs &a, float *rec)
    {
        const int d = a.c.head_dim;
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const float total = groups_sum(l[t]);
            const int row = 16 * t + c16;
            if (row >= a.rows)
                continue;
            if (g == 0) {
                rec[a.rows * d + row] = m[t];
                rec[a.rows * d + a.rows + row] = total;
            }
#pragma unroll
            for (int b = 0; b < NG; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e0 = (b * 16 + 4 * g + i) * VE;
                    if (e0 < d) {
#pragma unroll
                        for (int e = 0; e < VE; ++e)
                            rec[row * d + std::min(e0, d - VE) + e] = o[t][b * VE + e][i] * (1.0f / kLift);
                    }
                }
        }
    }
};

// The sum of parts of one row, and its weights' sum, relative to their largest maximum.
struct Joined {
    float sum, top, total;
};

template <typename T>
__device__ inline void write_row(const AttendArgs &a, int64_t seq, int unit, int row, int e, const Joined &x)
{
    const int head = unit / a.blocks, in_group = unit % a.blocks * a.rows + row;
    if (in_group >= a.group)
        return;
    const int64_t q = (int64_t)head * a.group + in_group;
    ((T *)(a.out + seq * a.o_seq + q * a.o_head))[e] = (T)(x.sum * inverse(x.total));
    if (a.lse && e == 0)
        a.lse[seq * a.q_heads + q] = log_sum(a, x.top, x.total);
}

__device__ inline int64_t uniform_i64(int64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(v & 0xffffffff)), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

template <typename T, int DP, int QT, bool PAGED>
__global__ void __launch_bounds__(64 * kAttendWaves) k_cache_attend(AttendArgs a)
{
    using A = Attend<T, DP, QT, PAGED>;
    constexpr int KT = A::KT, WAVES = kAttendWaves;
    extern __shared__ float records[];  // [waves][2]
    struct Part {
        int64_t u0, u1;  // the unit's tiles
        int32_t seq, unit, is, pad;
    };
    __shared__ Part parts[WAVES][2];
    const int wave = wave_id_uniform(), lane = lane_id();
    const int per_seq = a.c.heads * a.blocks;
    // the line's length
    int64_t sum = 0;
    for (int64_t i = lane; i < a.seqs; i += 64)
        sum += tiles_of<KT>(seen(a.c, a.window, i));
    const int64_t all = uniform_i64(wave_sum_i64(sum)) * per_seq, waves = (int64_t)gridDim.x * WAVES;
    const int64_t each = (all + waves - 1) / waves;
    const int64_t wg_begin = std::min(all, (int64_t)blockIdx.x * WAVES * each), wg_end = std::min(all, wg_begin + WAVES * each);
    const int64_t begin = std::min(all, wg_begin + wave * each), end = std::min(wg_end, begin + each);
    // the sequence that the stretch begins in
    int64_t seq = 0, at = 0;
    for (int64_t i0 = 0; i0 < a.seqs; i0 += 64) {
        int64_t n = i0 + lane < a.seqs ? (int64_t)tiles_of<KT>(seen(a.c, a.window, i0 + lane)) * per_seq : 0;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int64_t up = __shfl_up(n, m);
            if (lane >= m)
                n += up;
        }
        const unsigned long long past = __ballot(at + n > begin);
        if (past) {
            const int j = __ffsll(past) - 1;
            if (j > 0)
                at += __shfl(n, j - 1);
            seq = i0 + j;
            break;
        }
        at += __shfl(n, 63);
    }
    at = uniform_i64(at);
    int s32 = __builtin_amdgcn_readfirstlane((int)seq);
    if (lane < 2)
        parts[wave][lane].is = 0;
    A w;
    w.init(a);
    for (int64_t pos = begin; pos < end;) {
        const Seen s = seen(a.c, a.window, s32);
        const int nt = tiles_of<KT>(s);
        if (pos >= at + (int64_t)per_seq * nt) {
            at += (int64_t)per_seq * nt;
            ++s32;
            continue;
        }
        const int unit = (int)((pos - at) / nt);  // head * blocks + block
        const int64_t u0 = at + (int64_t)unit * nt, u1 = u0 + nt, stop = std::min(end, u1);
        const int head = unit / a.blocks, block = unit % a.blocks;
        w.begin(a, s32, head, block);
        const int32_t *const table = a.c.table + s32 * a.c.ld_table;
        const int first = s.first / KT * KT + (int)(pos - u0) * KT, n = (int)(stop - pos);
        for (int t = 0; t < n; ++t)
            w.tile(a, table, head, first + t * KT, s);
        if (pos == u0 && stop == u1) {
            w.finish(a, s32, head, block);
        } else {  // slot 0: it has begun before the stretch
            const int slot = pos == u0;
            w.leave(a, records + (wave * 2 + slot) * a.rec);
            if (lane == 0)
                parts[wave][slot] = {u0, u1, s32, unit, 1, 0};
        }
        pos = stop;
    }
    __syncthreads();
    // chains of parts: one of slot 1, or the first wavefront's of slot 0, and the slots 0 that follow while the unit goes on
    const int d = a.c.head_dim, elems = a.rows * d;
    bool goes_on = false;
    for (int p = 0; p < 2 * WAVES; ++p) {
        const int w0 = p / 2, slot = p % 2;
        if (!parts[w0][slot].is || (slot == 0 && w0 > 0))
            continue;
        const Part unit = parts[w0][slot];
        int n = 1;
        while (w0 + n < WAVES && wg_begin + (int64_t)(w0 + n) * each < std::min(unit.u1, wg_end))
            ++n;
        const bool whole = unit.u0 >= wg_begin && unit.u1 <= wg_end;
        float *const to = a.part + ((int64_t)blockIdx.x * 2 + (unit.u0 >= wg_begin)) * a.rec;
        goes_on |= unit.u0 >= wg_begin && unit.u1 > wg_end;
        for (int i = threadIdx.x; i < elems; i += 64 * WAVES) {
            const int row = i / d, e = i % d;
            Joined x = {0.0f, -INFINITY, 0.0f};
            for (int k = 0; k < n; ++k)
                x.top = fmaxf(x.top, records[((w0 + k) * 2 + (k == 0 ? slot : 0)) * a.rec + elems + row]);
            const float from = x.top == -INFINITY ? 0.0f : x.top;
            for (int k = 0; k < n; ++k) {
                const float *const r = records + ((w0 + k) * 2 + (k == 0 ? slot : 0)) * a.rec;
                const float f = exp2_fast((r[elems + row] - from) * a.factor);
                x.sum += r[i] * f;
                x.total += r[elems + a.rows + row] * f;
            }
            if (whole) {
                write_row<T>(a, unit.seq, unit.unit, row, e, x);
            } else {
                to[i] = x.sum;
                if (e == 0)
                    to[elems + row] = x.top, to[elems + a.rows + row] = x.total;
            }
        }
        if (goes_on && threadIdx.x == 0)
            a.tails[blockIdx.x] = {unit.seq, unit.unit, (int32_t)((unit.u1 - 1) / (WAVES * each))};
    }
    if (!goes_on && threadIdx.x == 0)
        a.tails[blockIdx.x].last = -1;
}

// Units that several workgroups have parts of: a workgroup for each that such a unit begins in, and for a share of its rows.
template <typename T>
__global__ void __launch_bounds__(256) k_cache_attend_join(AttendArgs a)
{
    __shared__ float sums[4][256];
    const int b = blockIdx.x, d = a.c.head_dim, elems = a.rows * d, wave = wave_id_uniform(), lane = lane_id();
    const Tail tail = a.tails[b];
    if (tail.last < 0)
        return;
    const int n = tail.last - b + 1;
    auto record = [&](int k) { return a.part + ((int64_t)(b + k) * 2 + (k == 0)) * a.rec; };
    for (int row = blockIdx.y; row < a.rows; row += gridDim.y) {
        Joined x = {0.0f, -INFINITY, 0.0f};
        for (int k = lane; k < n; k += 64)
            x.top = fmaxf(x.top, record(k)[elems + row]);
#pragma unroll
        for (int m = 1; m < 64; m *= 2)
            x.top = fmaxf(x.top, __shfl_xor(x.top, m));
        const float from = x.top == -INFINITY ? 0.0f : x.top;
        for (int k = lane; k < n; k += 64)
            x.total += record(k)[elems + a.rows + row] * exp2_fast((record(k)[elems + row] - from) * a.factor);
#pragma unroll
        for (int m = 1; m < 64; m *= 2)
            x.total += __shfl_xor(x.total, m);
        float acc[4] = {};
        for (int k = wave; k < n; k += 4) {
            const float *const r = record(k);
            const float f = exp2_fast((r[elems + row] - from) * a.factor);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (lane + 64 * j < d)
                    acc[j] += r[row * d + lane + 64 * j] * f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            sums[wave][lane + 64 * j] = acc[j];
        __syncthreads();
        const int e = threadIdx.x;
        if (e < d) {
            x.sum = (sums[0][e] + sums[1][e]) + (sums[2][e] + sums[3][e]);
            write_row<T>(a, tail.seq, tail.unit, row, e, x);
        }
        __syncthreads();
    }
}

struct AttendPlan {
    int qt, rows, blocks;
    int64_t rec;  // floats
    int wgs;
    int64_t tails;  // offset in the workspace
    size_t bytes;
};
AttendPlan attend_plan(const tig_cache &c, const tig_cache_attend &p)
{
    AttendPlan L = {};
    const int group = p.q_heads / c.heads, es = dtype_bytes(c.dtype), kt = es == 4 ? 16 : 32;
    L.qt = group > 16 && c.head_dim <= 128 ? 2 : 1;
    L.rows = std::min(group, 16 * L.qt);
    L.blocks = (group + 16 * L.qt - 1) / (16 * L.qt);
    L.rec = (int64_t)L.rows * (c.head_dim + 2);
    const int64_t cap = p.window > 0 ? std::min<int64_t>(p.window, (int64_t)c.max_pages * c.page_size) : (int64_t)c.max_pages * c.page_size;
    const int64_t tiles = p.seqs * c.heads * L.blocks * (cap / kt + 2);
    L.wgs = (int)std::min<int64_t>(1024, (tiles + kAttendWaves - 1) / kAttendWaves);
    L.tails = ((int64_t)L.wgs * 2 * L.rec * 4 + 255) / 256 * 256;
    L.bytes = (size_t)(L.tails + ((int64_t)L.wgs * sizeof(Tail) + 255) / 256 * 256);
    return L;
}

template <typename T, int DP, int QT, bool PAGED>
hipError_t launch_attend(const AttendArgs &a, const AttendPlan &L, hipStream_t s)
{
    const int lds = (int)(kAttendWaves * 2 * L.rec * 4);
    auto *const kernel = k_cache_attend<T, DP, QT, PAGED>;
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)L.wgs), dim3(64 * kAttendWaves), (unsigned)lds, s, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && L.wgs > 1) {
        hipLaunchKernelGGL((k_cache_attend_join<T>), dim3((unsigned)(L.wgs - 1), (unsigned)L.rows), dim3(256), 0, s, a);
        e = hipGetLastError();
    }
    return e;
}
template <typename T, int DP>
hipError_t launch_attend_dim(const AttendArgs &a, const AttendPlan &L, hipStream_t s)
{
    const bool paged = a.c.page_size % 16 == 0;
    if constexpr (DP <= 128)
        if (L.qt == 2)
            return paged ? launch_attend<T, DP, 2, true>(a, L, s) : launch_attend<T, DP, 2, false>(a, L, s);
    return paged ? launch_attend<T, DP, 1, true>(a, L, s) : launch_attend<T, DP, 1, false>(a, L, s);
}

int check_attend(const tig_cache *c, const tig_cache_attend *p)
{
    int rc = check_cache(c);
    if (rc != TIG_OK)
        return rc;
    if (!p || p->struct_size != sizeof(tig_cache_attend))
        return fail_text(TIG_EINVAL, "tig_cache_attend: NULL argument or wrong struct_size");
    if ((rc = check_sequences(*c, p->seqs, p->table, p->ld_table, p->lengths)) != TIG_OK)
        return rc;
    if (p->window < 0 || !(p->scale - p->scale == 0.0f))
        return fail_text(TIG_EINVAL, "tig_cache_attend: window is negative or scale is not finite");
    if (p->q_heads < 1 || p->q_heads > (1 << 14) || p->q_heads % c->heads)
        return fail_text(TIG_EINVAL, "tig_cache_attend: q_heads is no multiple of the cache's heads, or out of range");
    const int es = dtype_bytes(c->dtype);
    if (p->seqs > 0 && (!p->q || !p->out))
        return fail_text(TIG_EINVAL, "tig_cache_attend: q or out is NULL");
    if (!element_aligned(p->q, es) || !element_aligned(p->out, es) || !element_aligned(p->lse, 4))
        return fail_text(TIG_EINVAL, "tig_cache_attend: an address is not aligned to its element");
    for (const int64_t s : {p->q_seq, p->q_head, p->o_seq, p->o_head})
        if (s < 0 || s > ((int64_t)1 << 32))
            return fail_text(TIG_EINVAL, "tig_cache_attend: a stride is out of range");
    const int d = c->head_dim;
    const int64_t seq_span = (p->q_heads - 1) * p->o_head + d, head_span = (p->seqs - 1) * p->o_seq + d;
    if (p->seqs > 0 && ((p->seqs > 1 && p->o_seq < d) || (p->q_heads > 1 && p->o_head < d) ||
                        (p->seqs > 1 && p->q_heads > 1 && p->o_seq < seq_span && p->o_head < head_span)))
        return fail_text(TIG_EINVAL, "tig_cache_attend: rows of out overlap");
    return TIG_OK;
}

int check_attend_apart(const tig_cache &c, const tig_cache_attend &p)
{
    const int es = dtype_bytes(c.dtype);
    auto rows = [&](const void *x, int64_t seq, int64_t head) { return placed(x, {{p.seqs, seq}, {p.q_heads, head}}, c.head_dim, es); };
    const bool in_place = p.q == p.out && p.q_seq == p.o_seq && p.q_head == p.o_head;
    const int64_t n = p.seqs * p.q_heads;
    const Placed in[] = {rows(in_place ? nullptr : p.q, p.q_seq, p.q_head), placed_keys(c, c.k), placed_keys(c, c.v),
                         {p.table, p.seqs, c.max_pages, p.ld_table, 4}, {p.lengths, 1, p.seqs, p.seqs, 4}};
    const Placed out[] = {rows(p.out, p.o_seq, p.o_head), {p.lse, 1, n, n, 4}};
    return all_apart(in, out) ? TIG_OK : fail_text(TIG_EINVAL, "tig_cache_attend: an output overlaps another tensor of the call");
}

}  // namespace

}  // namespace tig

using namespace tig;

int tig_cache_attend_workspace_bytes(const tig_cache *cache, const tig_cache_attend *p, size_t *bytes)
{
    const int rc = check_attend(cache, p);
    if (rc != TIG_OK)
        return rc;
    if (!bytes)
        return fail_text(TIG_EINVAL, "tig_cache_attend_workspace_bytes: bytes is NULL");
    *bytes = p->seqs > 0 ? attend_plan(*cache, *p).bytes : 0;
    return TIG_OK;
}

int tig_cache_attend_run(const tig_cache *cache, const tig_cache_attend *p, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_attend(cache, p);
    if (rc != TIG_OK || p->seqs == 0)
        return rc;
    const AttendPlan L = attend_plan(*cache, *p);
    if (!workspace || ((uintptr_t)workspace & 255))
        return fail_text(TIG_EINVAL, "tig_cache_attend_run: workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < L.bytes)
        return fail_text(TIG_ENOSPACE, "tig_cache_attend_run: workspace too small");
    if ((rc = check_attend_apart(*cache, *p)) != TIG_OK)
        return rc;
    const int64_t es = dtype_bytes(cache->dtype);
    AttendArgs a = {};
    a.c = cache_view(*cache, p->table, p->ld_table, p->lengths);
    a.seqs = p->seqs, a.q = (const char *)p->q, a.out = (char *)p->out, a.lse = p->lse;
    a.q_seq = p->q_seq * es, a.q_head = p->q_head * es, a.o_seq = p->o_seq * es, a.o_head = p->o_head * es;
    a.q_heads = p->q_heads, a.group = p->q_heads / cache->heads, a.blocks = L.blocks, a.rows = L.rows, a.window = p->window;
    a.scale = p->scale;
    a.factor = std::max(std::fabs(p->scale) * 1.44269504f, FLT_MIN);  // (not zero: a masked score times it has to stay -infinity)
    a.flip = p->scale < 0.0f ? (es == 4 ? 0x80000000u : 0x80008000u) : 0u;
    a.part = (float *)workspace, a.tails = (Tail *)((char *)workspace + L.tails), a.rec = L.rec;
    const hipError_t e = with_dtype(cache->dtype, [&](auto t) {
        using T = decltype(t);
        if (cache->head_dim <= 64)
            return launch_attend_dim<T, 64>(a, L, (hipStream_t)hip_stream);
        if (cache->head_dim <= 128)
            return launch_attend_dim<T, 128>(a, L, (hipStream_t)hip_stream);
        return launch_attend_dim<T, 256>(a, L, (hipStream_t)hip_stream);
    });
    return e == hipSuccess ? TIG_OK : fail_global("tig_cache_attend_run", e);
}
