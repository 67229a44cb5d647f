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
// Weights P are 16-bit operands in two parts, P = hi + lo: the matrix units have the time (a tile of 32 keys of 128 columns takes a
// wavefront two microseconds and more from memory and a quarter of one for both parts), and one rounding of P would cost as much as rounding
// the output does.
//
// Bound by memory where there is much to read: 4 x 131071 rows of 8 heads of 128 columns in bf16, 64 query heads, 390 us (2.15 GB at 5.5 TB/s);
// 77 sequences of up to 4096 rows of 16 heads of 64 columns in fp16 129 us (655 MB, 5.1 TB/s); 4000 histories of up to 3000 rows of two heads of 50
// columns in fp32 236 us (1.14 GB, 4.8 TB/s).  Bound by its chain of reads (length, page, rows) and the two launches where there is
// little: one sequence of 1000 rows 15 us.
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
    int32_t together;                      // wavefronts of a workgroup that go through the same rows, each for another unit: 1, 2 or 4
    int32_t window;
    uint32_t flip;                         // sign bits of Q, to keep the factor positive
    float scale, factor;                   // scale; |scale| log2(e)
    float *part;                           // [workgroups x together x 2] records: rows x (head_dim + 2)
    struct Tail *tails;                    // [workgroups x together]
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
typedef const __attribute__((address_space(4))) int32_t ConstInt;  // (scalar loads: nothing that waits for them waits for rows on their way)
__device__ inline int seen_length(const CacheView &c, int seq)
{
    const int length = ((ConstInt *)(uintptr_t)c.lengths)[seq];
    return std::min(std::max(length, 0), c.capacity());
}
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
// What a unit takes beside its tiles, in tiles: it stands that much longer in the line, ahead of them.
constexpr int kUnitCost = 2;
constexpr int kNeverShared = 2;  // tiles of a unit that one wavefront takes in any case

// (a division in 64 bits is a hundred instructions)
__device__ inline int64_t quotient(int64_t a, int64_t b) { return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b; }

// sums over the lanes up to and with each
__device__ inline int64_t wave_scan_i64(int64_t v)
{
    if (!__any((v >> 25) != 0)) {  // (within rows of sixteen lanes, then the rows' sums carried on)
        int x = (int)v;
        x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
        x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
        x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
        return x;
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int64_t up = __shfl_up(v, m);
        if (lane_id() >= m)
            v += up;
    }
    return v;
}

__device__ inline int64_t uniform_i64(int64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(v & 0xffffffff)), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// maximum over the four lanes that share lane % 16
__device__ inline float groups_max(float v)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// of a sum of weights; nothing was there: 0
__device__ inline float inverse(float total) { return total == 0.0f ? 0.0f : 1.0f / total; }
__device__ inline float log_sum(const AttendArgs &a, float top, float total) { return total == 0.0f ? -INFINITY : top * fabsf(a.scale) + logf(total); }

template <typename T, int DP, int QT, bool PAGED>
struct Attend {
    using Type = T;
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
    int k_off[NKB];                // byte of the lane's piece of a key (PAGED: of sixteen rows of keys; outside of them: none)
    int v_off[PAGED ? 4 : 1][NG];  // ... of values
    intx4 tail;                    // of the lane's piece of the last block: nothing behind the row, once what two pieces have
    // per unit
    intx4 qv[QT][NKB];
    // per tile
    intx4 kv[NS][NKB];
    Vpiece vv[VK][NG];
    int64_t from[NS];              // where each sixteen rows lie; not PAGED: where the lane's row of them does, -1: nowhere
    int extent[NS];                // bytes there (PAGED)
    float m[QT], l[QT];
    floatx4 o[QT][NG * VE];

    __device__ inline void init(const AttendArgs &a)
    {
        lane = lane_id(), c16 = lane % 16, g = lane / 16;
        const int d = a.c.head_dim, stride = (int)a.c.token_stride;
        constexpr int kNone = PAGED ? 0x40000000 : 0;  // (no sixteen rows are that long)
#pragma unroll
        for (int b = 0; b < NKB; ++b) {
            const int e = (b * 4 + g) * PE;
            k_off[b] = e >= d ? kNone : (PAGED ? c16 * stride : 0) + std::min(e, d - PE) * ES;
        }
        const int e0 = ((d - 1) / (4 * PE) * 4 + g) * PE, dup = e0 + PE - d;  // elements of a last piece that the one before has as well
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (ES == 4)
                tail[i] = i < dup ? 0 : -1;
            else
                tail[i] = 2 * i + 1 < dup ? 0 : 2 * i < dup ? (int)0xffff0000 : -1;
        }
        if (e0 >= d)
            tail = intx4{0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < NG; ++b) {
            const int e = (b * 16 + c16) * VE;
#pragma unroll
            for (int i = 0; i < (PAGED ? 4 : 1); ++i)
                v_off[i][b] = e >= d ? kNone : (PAGED ? (4 * g + i) * stride : 0) + std::min(e, d - VE) * ES;
        }
    }
    // what of the b-th blocks' pieces a row has: all, nothing, or in the last block that it reaches into what `tail` keeps
    __device__ inline intx4 within(intx4 x, int b, int d) const
    {
        const int last = (d - 1) / (4 * PE);
        return b < last ? x : b == last ? x & tail : intx4{0, 0, 0, 0};
    }
    // A unit's queries: asked for here, taken at its first tile.
    __device__ inline void load_queries(const AttendArgs &a, int seq, int head, int block)
    {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int row = block * 16 * QT + 16 * t + c16;
            const char *const p = a.q + seq * a.q_seq + (int64_t)(head * a.group + std::min(row, a.group - 1)) * a.q_head;
#pragma unroll
            for (int b = 0; b < NKB; ++b)
                qv[t][b] = ((const Sixteen *)(p + std::min((b * 4 + g) * PE, a.c.head_dim - PE) * ES))->v;
        }
    }
    __device__ inline void start(const AttendArgs &a, int block)
    {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const uint32_t keep = block * 16 * QT + 16 * t + c16 < a.group ? 0xffffffffu : 0u;
#pragma unroll
            for (int b = 0; b < NKB; ++b) {
                asm volatile("" : "+v"(qv[t][b]));
                qv[t][b] = within(qv[t][b], b, a.c.head_dim);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    qv[t][b][i] = (qv[t][b][i] ^ a.flip) & keep;
            }
            m[t] = -INFINITY, l[t] = 0.0f;
#pragma unroll
            for (int i = 0; i < NG * VE; ++i)
                o[t][i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }

    // Where rows base .. base + KT - 1 of the sequence lie: asked for two tiles ahead.  PAGED: the page of each sixteen rows, else the
    // one of the lane's row of each sixteen; -1: none.
    struct Pages {
        int page[NS];
    };
    __device__ inline Pages no_pages() const
    {
        Pages x;
#pragma unroll
        for (int t = 0; t < NS; ++t)
            x.page[t] = -1;
        return x;
    }
    __device__ inline Pages pages(const CacheView &c, const int32_t *table, int base, const Seen &s) const
    {
        Pages x;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            if constexpr (PAGED) {
                const int at = base + 16 * t;
                x.page[t] = -1;
                if (at < s.end)
                    x.page[t] = ((ConstInt *)(uintptr_t)table)[c.div.quotient(at)];
            } else {  // (no choice between the load and another value: it would become a branch; an empty sequence reads its table's first entry)
                const int key = base + 16 * t + c16;
                x.page[t] = table[c.div.quotient(std::max(0, std::min(std::max(key, s.first), s.end - 1)))] | (key >= s.first && key < s.end ? 0 : -1);
            }
        }
        return x;
    }
    // ... and as offsets from the head's first row
    __device__ inline void resolve(const CacheView &c, const Pages &where, int base, const Seen &s)
    {
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            const int at = base + 16 * t + (PAGED ? 0 : c16), page = where.page[t];
            const bool ok = c.page_ok(page);
            from[t] = ok ? page * c.page_stride + (at - c.div.quotient(at) * c.page_size) * c.token_stride : PAGED ? 0 : -1;
            if constexpr (PAGED)  // rows behind the end lie outside of the extent and read as zero, where there is no page all do
                extent[t] = ok ? (std::min(16, s.end - at) - 1) * (int)c.token_stride + c.head_dim * ES : 0;
        }
    }

    // The tile's keys: rows base .. base + KT - 1 of the sequence, as resolved.  PAGED: a descriptor for sixteen rows, the lane's
    // offsets are the same for every tile.  Else each row by itself; one that is not there reads another one's memory and counts nothing.
    __device__ inline void load_keys(const char *rows)
    {
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            if constexpr (PAGED) {
                const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(rows + from[t]), 0, extent[t], kBufferFlags);
#pragma unroll
                for (int b = 0; b < NKB; ++b)
                    kv[t][b] = __builtin_bit_cast(intx4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, k_off[b], 0, 0));
            } else {
                const char *const p = rows + std::max<int64_t>(from[t], 0);
#pragma unroll
                for (int b = 0; b < NKB; ++b)
                    kv[t][b] = ((const Sixteen *)(p + k_off[b]))->v;
            }
        }
    }
    // ... and its values
    __device__ inline void load_values(const char *rows)
    {
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            if constexpr (PAGED) {
                const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(rows + from[t]), 0, extent[t], kBufferFlags);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int b = 0; b < NG; ++b) {
                        if constexpr (VE * ES == 16)
                            vv[4 * t + i][b] = __builtin_bit_cast(Vpiece, __builtin_amdgcn_raw_buffer_load_b128(rsrc, v_off[i][b], 0, 0));
                        else
                            vv[4 * t + i][b] = __builtin_bit_cast(Vpiece, __builtin_amdgcn_raw_buffer_load_b64(rsrc, v_off[i][b], 0, 0));
                    }
            } else {
                struct __attribute__((packed, aligned(2))) Any {
                    Vpiece v;
                };
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const char *const p = rows + std::max<int64_t>(__shfl(from[t], 4 * g + i), 0);
#pragma unroll
                    for (int b = 0; b < NG; ++b)
                        vv[4 * t + i][b] = ((const Any *)(p + v_off[0][b]))->v;
                }
            }
        }
    }

    // The keys as they are multiplied.  (A load's value is used whatever the conditions: else it would move into a branch, and be waited
    // for there.)
    __device__ inline void take_keys(int d)
    {
        if (PAGED ? d % PE != 0 : d < DP) {
#pragma unroll
            for (int t = 0; t < NS; ++t)
#pragma unroll
                for (int b = 0; b < NKB; ++b) {
                    if constexpr (!PAGED)
                        asm volatile("" : "+v"(kv[t][b]));
                    kv[t][b] = within(kv[t][b], b, d);
                }
        }
    }
    // ... and the values; cut: those of keys that do not count are zero (zero times what no sequence has is not zero where that is
    // infinite)
    template <class F>
    __device__ inline void take_values(bool cut, F &&valid)
    {
        if constexpr (!PAGED) {
#pragma unroll
            for (int i = 0; i < VK; ++i)
#pragma unroll
                for (int b = 0; b < NG; ++b)
#pragma unroll
                    for (int e = 0; e < VE * ES / 4; ++e)
                        asm volatile("" : "+v"(vv[i][b].d[e]));
        }
        if (cut) {
#pragma unroll
            for (int i = 0; i < VK; ++i)
#pragma unroll
                for (int b = 0; b < NG; ++b)
#pragma unroll
                    for (int e = 0; e < VE * ES / 4; ++e)
                        vv[i][b].d[e] = valid(i) ? vv[i][b].d[e] : 0;
        }
    }

    // A tile, of this unit or the next one's first.
    struct Next {
        Pages pages;
        const char *keys, *values;  // the head's first row
        int base;
        Seen s;
        int seq, head, block;       // seq >= 0: another unit, whose queries are wanted too
    };

    // A tile whose keys and values are on their way; those of the next one are asked for as soon as the registers are free.
    __device__ inline void tile(const AttendArgs &a, int base, const Seen &s, const Next &next)
    {
        const CacheView &c = a.c;
        const int d = c.head_dim;
        take_keys(d);
        float p[QT][VK];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int u = 0; u < NS; ++u) {
                floatx4 sc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int b = 0; b < NKB; ++b)
                    mma16(sc, kv[u][b], qv[t][b], T());
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    p[t][4 * u + i] = sc[i];
            }
        // which of the lane's four (eight) keys are there; whole: all keys of the tile
        bool whole = base >= s.first && base + KT <= s.end;
        unsigned long long there[NS];
#pragma unroll
        for (int u = 0; u < NS; ++u) {
            there[u] = PAGED ? (extent[u] > 0 ? ~0ull : 0ull) : __ballot(from[u] >= 0);
            whole = whole && there[u] == ~0ull;
        }
        auto valid = [&](int i) {
            const int key = base + 16 * (i / 4) + 4 * g + i % 4;
            return (PAGED ? there[i / 4] != 0 && key >= s.first && key < s.end : (there[i / 4] >> (4 * g + i % 4)) & 1);
        };
        resolve(c, next.pages, next.base, next.s);
        load_keys(next.keys);
        if (next.seq >= 0)
            load_queries(a, next.seq, next.head, next.block);
        if (!whole) {
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
                for (int i = 0; i < VK; ++i)
                    p[t][i] = valid(i) ? p[t][i] : -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            float top = p[t][0];
#pragma unroll
            for (int i = 1; i < VK; ++i)
                top = fmaxf(top, p[t][i]);
            top = fmaxf(m[t], groups_max(top));
            const float from = top == -INFINITY ? 0.0f : top;
            if (__any(top > m[t])) {  // (most tiles of a long sequence bring no new maximum)
                const float keep = exp2_fast((m[t] - from) * a.factor);  // (another lane's may be new where this one's is still -infinity)
                l[t] *= keep;
#pragma unroll
                for (int i = 0; i < NG * VE; ++i)
                    o[t][i] *= keep;
                m[t] = top;
            }
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < VK; ++i) {
                p[t][i] = exp2_fast((p[t][i] - from) * a.factor);
                sum += p[t][i];
            }
            l[t] += sum;
        }
        take_values(PAGED ? base < s.first : !whole, valid);
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
        load_values(next.values);
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

// fp32 with one or two query heads to a head: sixteen queries' products of which one is wanted take the matrix units a thousand cycles a tile
// of 16 keys and 64 columns, that one in vector instructions a tenth of it (4000 histories of two heads of 50 columns, 1.14 GB: 260 and
// 236 us).  The lanes have keys and values as above; the scores' sums over a lane's columns are joined over the four lanes of a key, each
// lane then weighs its key, and the weights of a lane's four keys of values are fetched from the lanes that have them.
template <int DP, int G, bool PAGED>
struct AttendFew : Attend<float, DP, 1, PAGED> {
    using Base = Attend<float, DP, 1, PAGED>;
    using Base::c16, Base::g, Base::kv, Base::vv, Base::from, Base::extent;
    static constexpr int NKB = Base::NKB, NG = Base::NG, VE = Base::VE, KT = Base::KT, kColumns = NG * VE;
    static_assert(KT == 16 && VE == 4, "");

    floatx4 q[G][NKB];
    float m[G], l[G], o[G][kColumns];  // m: all lanes alike; l: of the lane's key; o: of the lane's keys of values

    __device__ inline void load_queries(const AttendArgs &a, int seq, int head, int)
    {
#pragma unroll
        for (int t = 0; t < G; ++t) {
            const char *const p = a.q + seq * a.q_seq + (int64_t)(head * a.group + std::min(t, a.group - 1)) * a.q_head;
#pragma unroll
            for (int b = 0; b < NKB; ++b)
                q[t][b] = __builtin_bit_cast(floatx4, ((const Sixteen *)(p + std::min((b * 4 + g) * 4, a.c.head_dim - 4) * 4))->v);
        }
    }
    __device__ inline void start(const AttendArgs &a, int)
    {
#pragma unroll
        for (int t = 0; t < G; ++t) {
#pragma unroll
            for (int b = 0; b < NKB; ++b) {
                intx4 x = __builtin_bit_cast(intx4, q[t][b]);
                asm volatile("" : "+v"(x));
                x = this->within(x, b, a.c.head_dim);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[i] ^= a.flip;
                q[t][b] = __builtin_bit_cast(floatx4, x);
            }
            m[t] = -INFINITY, l[t] = 0.0f;
#pragma unroll
            for (int i = 0; i < kColumns; ++i)
                o[t][i] = 0.0f;
        }
    }
    __device__ inline void tile(const AttendArgs &a, int base, const Seen &s, const typename Base::Next &next)
    {
        const CacheView &c = a.c;
        const int d = c.head_dim;
        this->take_keys(d);
        float sc[G];
#pragma unroll
        for (int t = 0; t < G; ++t) {
            floatx4 part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int b = 0; b < NKB; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    part[i] = fmaf(__int_as_float(kv[0][b][i]), q[t][b][i], part[i]);
            sc[t] = groups_sum((part[0] + part[1]) + (part[2] + part[3]));
        }
        const int key = base + c16;
        const bool here = PAGED ? extent[0] > 0 && key >= s.first && key < s.end : from[0] >= 0;
        const unsigned long long there = __ballot(here);
        const bool whole = there == ~0ull, cut = PAGED ? base < s.first : !whole;
        this->resolve(c, next.pages, next.base, next.s);
        this->load_keys(next.keys);
        if (next.seq >= 0)
            load_queries(a, next.seq, next.head, next.block);
        float p[G][4];
#pragma unroll
        for (int t = 0; t < G; ++t) {
            if (!whole)
                sc[t] = here ? sc[t] : -INFINITY;
            const float top = fmaxf(m[t], row_max_all(sc[t]));
            if (__any(top > m[t])) {
                const float keep = exp2_fast((m[t] - top) * a.factor);
                l[t] *= keep;
#pragma unroll
                for (int i = 0; i < kColumns; ++i)
                    o[t][i] *= keep;
                m[t] = top;
            }
            const float w = exp2_fast((sc[t] - (top == -INFINITY ? 0.0f : top)) * a.factor);
            l[t] += w;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                p[t][i] = __shfl(w, 4 * g + i);
        }
        this->take_values(cut, [&](int i) { return (there >> (4 * g + i)) & 1; });
#pragma unroll
        for (int t = 0; t < G; ++t)
#pragma unroll
            for (int b = 0; b < NG; ++b)
#pragma unroll
                for (int e = 0; e < VE; ++e)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        o[t][b * VE + e] = fmaf(p[t][i], __int_as_float(vv[i][b].d[e]), o[t][b * VE + e]);
        this->load_values(next.values);
    }
    // f(row, first column, the lane's four columns): each column of each row once
    template <class F>
    __device__ inline void columns(const AttendArgs &a, F &&f)
    {
#pragma unroll
        for (int t = 0; t < G; ++t) {
#pragma unroll
            for (int b = 0; b < NG; ++b) {
                floatx4 x;
#pragma unroll
                for (int e = 0; e < VE; ++e)
                    x[e] = groups_sum(o[t][b * VE + e]);
                const int e0 = (b * 16 + c16) * VE;
                if (t < a.group && b % 4 == g && e0 < a.c.head_dim)
                    f(t, std::min(e0, a.c.head_dim - VE), x);
            }
        }
    }
    __device__ inline void finish(const AttendArgs &a, int64_t seq, int head, int)
    {
        float by[G];
#pragma unroll
        for (int t = 0; t < G; ++t) {
            const float total = row_sum_all(l[t]);
            by[t] = inverse(total);
            if (a.lse && t < a.group && this->lane == 0)
                a.lse[seq * a.q_heads + head * a.group + t] = log_sum(a, m[t], total);
        }
        columns(a, [&](int t, int e, const floatx4 &x) {
            float r = by[0];
#pragma unroll
            for (int i = 1; i < G; ++i)
                r = t == i ? by[i] : r;
            store_four((float *)(a.out + seq * a.o_seq + (int64_t)(head * a.group + t) * a.o_head) + e, x * r, 4);
        });
    }
    __device__ inline void leave(const AttendArgs &a, float *rec)
    {
        const int elems = a.rows * a.c.head_dim;
#pragma unroll
        for (int t = 0; t < G; ++t) {
            const float total = row_sum_all(l[t]);
            if (t < a.group && this->lane == 0)
                rec[elems + t] = m[t], rec[elems + a.rows + t] = total;
        }
        columns(a, [&](int t, int e, const floatx4 &x) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                rec[t * a.c.head_dim + e + i] = x[i];
        });
    }
};

// no tile of a unit
__device__ inline void leave_nothing(const AttendArgs &a, float *rec)
{
    const int elems = a.rows * a.c.head_dim;
    for (int i = lane_id(); i < elems + 2 * a.rows; i += 64)
        rec[i] = i >= elems && i < elems + a.rows ? -INFINITY : 0.0f;
}

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

// SOLO: a workgroup for each unit, and no line.
template <class A, int WAVES, bool SOLO>
__global__ void __launch_bounds__(64 * WAVES) k_cache_attend(AttendArgs a)
{
    using T = typename A::Type;
    constexpr int KT = A::KT, kCost = SOLO ? 0 : kUnitCost;
    auto place_of = [&](const Seen &s) { return tiles_of<KT>(s) + kCost; };
    extern __shared__ float records[];  // [waves][2]
    struct Part {
        int64_t u0, u1;  // the unit's tiles
        int32_t seq, unit, is, pad;
    };
    __shared__ Part parts[WAVES][2];
    const int wave = wave_id_uniform(), lane = lane_id();
    const int units = a.c.heads * a.blocks, together = SOLO ? 1 : a.together, strides = WAVES / together;  // stretches of a workgroup
    const int mine = wave % together, stretch = wave / together;
    const int per_seq = (units + together - 1) / together;
    const int64_t waves = (int64_t)gridDim.x * strides;
    int64_t all, at = 0, each, wg_begin, wg_end, begin, end;  // the line and the stretch of it; at: where sequence s32 begins
    int s32 = 0;
    auto deal = [&]() {
        each = quotient(all + waves - 1, waves);
        wg_begin = std::min(all, (int64_t)blockIdx.x * strides * each), wg_end = std::min(all, wg_begin + strides * each);
        begin = std::min(all, wg_begin + stretch * each), end = std::min(wg_end, begin + each);
    };
    // among sequences s32 + lane, the one that the stretch begins in
    auto find = [&](int n_here, int64_t scan) {  // scan: tiles up to and with the lane's sequence, from `at` on
        const unsigned long long past = __ballot(lane < n_here && at + scan > begin);
        const int j = past ? __ffsll(past) - 1 : 0;
        if (j > 0)
            at = uniform_i64(at + __shfl(scan, j - 1));
        s32 = __builtin_amdgcn_readfirstlane(s32 + j);
        return past != 0;
    };
    if constexpr (SOLO) {
        s32 = blockIdx.x / units;
        all = place_of(seen(a.c, a.window, s32));
        at = -(int64_t)(blockIdx.x - s32 * units) * all;  // (the unit begins at 0)
        each = (int)(all + WAVES - 1) / WAVES;
        wg_begin = 0, wg_end = all, begin = std::min(all, wave * each), end = std::min(all, begin + each);
    } else if (a.seqs <= 64) {
        const int64_t scan = wave_scan_i64(lane < a.seqs ? (int64_t)place_of(seen(a.c, a.window, lane)) * per_seq : 0);
        all = uniform_i64(__shfl(scan, 63));
        deal();
        find((int)a.seqs, scan);
    } else {  // the wavefronts add ranges of sequences up; then the range, then the sequence
        constexpr int kRanges = 256;
        __shared__ int64_t ranges[kRanges];
        const int blocks = (int)((a.seqs + 63) / 64), span = (blocks + kRanges - 1) / kRanges;  // a range: `span` times 64 sequences
        const int n_ranges = (blocks + span - 1) / span;
        for (int r = wave; r < n_ranges; r += WAVES) {
            int64_t sum = 0;
            for (int i = r * span * 64 + lane, end = std::min<int64_t>(a.seqs, (r + 1) * (int64_t)span * 64); i < end; i += 64)
                sum += place_of(seen(a.c, a.window, i));
#pragma unroll
            for (int m = 1; m < 64; m *= 2)
                sum += __shfl_xor(sum, m);
            if (lane == 0)
                ranges[r] = sum * per_seq;
        }
        __syncthreads();
        int64_t scan[kRanges / 64];
        all = 0;
#pragma unroll
        for (int i = 0; i < kRanges / 64; ++i) {
            scan[i] = 0;
            if (64 * i < n_ranges) {
                scan[i] = all + wave_scan_i64(64 * i + lane < n_ranges ? ranges[64 * i + lane] : 0);
                all = uniform_i64(__shfl(scan[i], 63));
            }
        }
        deal();
        bool found = false;
#pragma unroll
        for (int i = 0; i < kRanges / 64; ++i) {
            const unsigned long long past = __ballot(64 * i + lane < n_ranges && scan[i] > begin);
            if (past && !found) {
                found = true;
                const int r = 64 * i + __ffsll(past) - 1;
                at = r > 0 ? __shfl(r % 64 > 0 ? scan[i] : scan[std::max(i - 1, 0)], (r - 1) % 64) : 0;
                s32 = r * span * 64;
            }
        }
        at = uniform_i64(at), s32 = __builtin_amdgcn_readfirstlane(s32);
        const int s_end = (int)std::min<int64_t>(a.seqs, s32 + span * 64);
        while (begin < end && s32 < s_end) {
            const int n = std::min(64, s_end - s32);
            const int64_t within = wave_scan_i64(lane < n ? (int64_t)place_of(seen(a.c, a.window, s32 + lane)) * per_seq : 0);
            if (find(n, within))
                break;
            at = uniform_i64(at + __shfl(within, 63)), s32 += n;
        }
    }
    if (lane < 2)
        parts[wave][lane].is = 0;
    A w;
    w.init(a);
    // The units of the stretch, one ahead of the one that is worked on.
    struct Unit {
        int64_t u0, u1;  // its place in the line
        Seen s;          // what it sees
        int seq, unit, head, block, base, n;  // first row and number of the tiles that are the stretch's; n < 0: there is no such unit
        bool begins, ends;
    };
    // Units that are short beside the stretches are not shared, nor are units of two tiles (2059 sequences of one row: 40 us shared, 27 not): the
    // stretches differ by a sixteenth for it.
    const int short_unit = (int)std::min<int64_t>(1 << 20, std::max<int64_t>(each / 16 + 1, kNeverShared)) + kCost;
    int64_t pos = begin;
    const int last_seq = (int)a.seqs - 1;
    int length = seen_length(a.c, s32), next_length = seen_length(a.c, std::min(s32 + 1, last_seq));  // (asked for a unit ahead)
    auto advance = [&]() {
        Unit u;
        u.n = -1;
        while (pos < end) {
            const Seen s = {a.window > 0 ? std::max(0, length - a.window) : 0, length};
            const int place = place_of(s);
            if (pos >= at + (int64_t)per_seq * place) {
                at += (int64_t)per_seq * place;
                length = next_length, next_length = seen_length(a.c, std::min(++s32 + 1, last_seq));
                continue;
            }
            const int turn = (int)quotient(pos - at, place);
            u.unit = turn * together + mine;  // head * blocks + block
            u.u0 = at + (int64_t)turn * place, u.u1 = u.u0 + place;
            int64_t stop = std::min(end, u.u1);
            if (!SOLO && place <= short_unit) {  // whole, in the stretch that it begins in
                if (pos > u.u0) {
                    pos = stop;
                    continue;
                }
                stop = u.u1;
            }
            const int from = std::max(0, (int)(pos - u.u0) - kCost), to = std::max(0, (int)(stop - u.u0) - kCost);
            u.begins = pos == u.u0, u.ends = stop == u.u1;
            pos = stop;
            if (u.unit >= units)
                continue;
            u.seq = s32, u.s = s, u.head = u.unit / a.blocks, u.block = u.unit - u.head * a.blocks;
            if (to == from) {  // none of its tiles: a part all the same, so that the parts of a unit follow each other
                leave_nothing(a, records + (wave * 2 + u.begins) * a.rec);
                if (lane == 0)
                    parts[wave][u.begins] = {u.u0, u.u1, u.seq, u.unit, 1, 0};
                continue;
            }
            u.n = to - from, u.base = s.first / KT * KT + from * KT;
            u.s.end = std::min(s.end, u.base + u.n * KT);  // (nothing is asked for behind the stretch)
            break;
        }
        return u;
    };
    auto table_of = [&](const Unit &u) { return a.c.table + u.seq * a.c.ld_table; };
    auto keys_of = [&](const Unit &u) { return a.c.k + u.head * a.c.head_stride; };
    auto values_of = [&](const Unit &u) { return a.c.v + u.head * a.c.head_stride; };
    Unit u = advance();
    if (u.n > 0) {
        w.resolve(a.c, w.pages(a.c, table_of(u), u.base, u.s), u.base, u.s);
        w.load_keys(keys_of(u));
        w.load_queries(a, u.seq, u.head, u.block);
        w.load_values(values_of(u));
    }
    while (u.n > 0) {
        typename A::Pages ahead = w.pages(a.c, table_of(u), u.base + KT, u.s);
        const Unit v = advance();
        typename A::Next other = {{}, keys_of(u), values_of(u), u.base, {0, 0}, -1, 0, 0};  // (nothing, where there is no other unit)
        if (v.n > 0)
            other = {w.pages(a.c, table_of(v), v.base, v.s), keys_of(v), values_of(v), v.base, v.s, v.seq, v.head, v.block};
        else
            other.pages = w.no_pages();
        w.start(a, u.block);
        const char *const keys = keys_of(u), *const values = values_of(u);
        const int32_t *const table = table_of(u);
        for (int t = 0; t < u.n - 1; ++t) {
            const typename A::Pages then = w.pages(a.c, table, u.base + (t + 2) * KT, u.s);
            w.tile(a, u.base + t * KT, u.s, {ahead, keys, values, u.base + (t + 1) * KT, u.s, -1, 0, 0});
            ahead = then;
        }
        w.tile(a, u.base + (u.n - 1) * KT, u.s, other);
        if (u.begins && u.ends) {
            w.finish(a, u.seq, u.head, u.block);
        } else {  // slot 0: it has begun before the stretch
            w.leave(a, records + (wave * 2 + u.begins) * a.rec);
            if (lane == 0)
                parts[wave][u.begins] = {u.u0, u.u1, u.seq, u.unit, 1, 0};
        }
        u = v;
    }
    __syncthreads();
    // chains of parts: one of slot 1, or a stretch's first one of slot 0, and the slots 0 that follow while the unit goes on
    const int d = a.c.head_dim, elems = a.rows * d;
    int goes_on = 0;
    unsigned long long starts = __ballot(lane < 2 * WAVES && parts[lane / 2 % WAVES][lane % 2].is && (lane % 2 == 1 || lane / 2 < together));
    while (starts) {
        const int p = __ffsll(starts) - 1, w0 = p / 2, slot = p % 2;
        starts &= starts - 1;
        const Part unit = parts[w0][slot];
        int n = 1;
        while (w0 + n * together < WAVES && wg_begin + (int64_t)(w0 / together + n) * each < std::min(unit.u1, wg_end))
            ++n;
        const bool whole = unit.u0 >= wg_begin && unit.u1 <= wg_end, first = unit.u0 >= wg_begin;
        const int64_t line = (int64_t)blockIdx.x * together + w0 % together;
        float *const to = a.part + (line * 2 + first) * a.rec;
        auto record = [&](int k) { return records + ((w0 + k * together) * 2 + (k == 0 ? slot : 0)) * a.rec; };
        for (int row = wave; row < a.rows; row += WAVES) {
            float m[WAVES], l[WAVES];
            Joined x = {0.0f, -INFINITY, 0.0f};
#pragma unroll
            for (int k = 0; k < WAVES; ++k) {
                const float *const r = record(std::min(k, n - 1)) + elems + row;
                m[k] = k < n ? r[0] : -INFINITY, l[k] = k < n ? r[a.rows] : 0.0f;
                x.top = fmaxf(x.top, m[k]);
            }
            const float from = x.top == -INFINITY ? 0.0f : x.top;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) {
                m[k] = exp2_fast((m[k] - from) * a.factor);
                x.total += l[k] * m[k];
            }
            for (int e = lane; e < d; e += 64) {
                x.sum = 0.0f;
#pragma unroll
                for (int k = 0; k < WAVES; ++k)
                    if (k < n)
                        x.sum += record(k)[row * d + e] * m[k];
                if (whole)
                    write_row<T>(a, unit.seq, unit.unit, row, e, x);
                else
                    to[row * d + e] = x.sum;
            }
            if (!whole && lane == 0)
                to[elems + row] = x.top, to[elems + a.rows + row] = x.total;
        }
        if (first && !whole) {
            goes_on |= 1 << w0 % together;
            if (threadIdx.x == 0)
                a.tails[line] = {unit.seq, unit.unit, (int32_t)quotient(unit.u1 - 1, strides * each)};
        }
    }
    if (!SOLO && (int)threadIdx.x < together && !(goes_on >> threadIdx.x & 1))
        a.tails[(int64_t)blockIdx.x * together + threadIdx.x].last = -1;
}

// Units that several workgroups have parts of: those that begin in four workgroups' stretches, one row of them.  A unit of up to
// four parts is one wavefront's, of the others' parts each of the four takes every fourth.  Sixty-four parts at a time: their maxima and sums
// are a lane's each, while the first rows are on their way.
template <typename T>
__global__ void __launch_bounds__(256) k_cache_attend_join(AttendArgs a, int lines)
{
    constexpr int kDeep = 8;
    __shared__ float sums[4][256], tops[4], totals[4];
    const int d = a.c.head_dim, elems = a.rows * d, wave = wave_id_uniform(), lane = lane_id(), row = blockIdx.y;
    auto join = [&](int b, const Tail &tail, int k0, int step, float (&acc)[4]) {
        const int n = (tail.last - b / a.together + step - k0) / step;  // parts k0, k0 + step, ..
        auto record = [&](int k) { return a.part + ((int64_t)(b + (k0 + k * step) * a.together) * 2 + (k0 + k * step == 0)) * a.rec; };
        Joined x = {0.0f, -INFINITY, 0.0f};
        for (int first = 0; first < n; first += 64) {
            const int left = std::min(64, n - first);
            const float *const mine = record(first + std::min(lane, left - 1)) + elems + row;
            float m = mine[0], l = mine[a.rows];
            if (lane >= left)
                m = -INFINITY, l = 0.0f;
            const float top = fmaxf(wave_max_all(m), x.top);
            const float from = top == -INFINITY ? 0.0f : top;
            const float f = exp2_fast((m - from) * a.factor), keep = exp2_fast((x.top - from) * a.factor);
            x.total = x.total * keep + wave_sum_all(l * f);
            x.top = top;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[j] *= keep;
            for (int k = 0; k < left; k += kDeep) {
                float r[kDeep][4];
#pragma unroll
                for (int i = 0; i < kDeep; ++i) {
                    const float *const p = record(first + std::min(k + i, left - 1)) + row * d;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (64 * j < d)
                            r[i][j] = p[std::min(lane + 64 * j, d - 1)];
                }
#pragma unroll
                for (int i = 0; i < kDeep; ++i) {
                    if (k + i >= left)
                        break;
                    const float by = __shfl(f, k + i);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (64 * j < d)
                            acc[j] += r[i][j] * by;
                }
            }
        }
        return x;
    };
    Tail tails[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int b = blockIdx.x * 4 + i;
        tails[i] = a.tails[std::min(b, lines - 1)];
        if (b >= lines)
            tails[i].last = -1;
    }
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
        const int b = blockIdx.x * 4 + i;
        const Tail tail = i == 0 ? tails[0] : i == 1 ? tails[1] : i == 2 ? tails[2] : tails[3];
        if (tail.last < 0)
            continue;
        const bool alone = tail.last - b / a.together < 4;
        if (alone && wave != i)
            continue;
        float acc[4] = {};
        Joined x = join(b, tail, alone ? 0 : wave, alone ? 1 : 4, acc);
        if (alone) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (lane + 64 * j < d) {
                    x.sum = acc[j];
                    write_row<T>(a, tail.seq, tail.unit, row, lane + 64 * j, x);
                }
            continue;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            sums[wave][lane + 64 * j] = acc[j];
        if (lane == 0)
            tops[wave] = x.top, totals[wave] = x.total;
        __syncthreads();
        const int e = threadIdx.x;
        if (e < d) {
            x = {0.0f, fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), 0.0f};
            const float from = x.top == -INFINITY ? 0.0f : x.top;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = exp2_fast((tops[w] - from) * a.factor);
                x.sum += sums[w][e] * f;
                x.total += totals[w] * f;
            }
            write_row<T>(a, tail.seq, tail.unit, row, e, x);
        }
        __syncthreads();
    }
}

struct AttendPlan {
    int few, qt, rows, blocks;
    int64_t rec;  // floats
    int wgs, together;
    bool solo, joins;
    int64_t tails;  // offset in the workspace
    size_t bytes;
};
AttendPlan attend_plan(const tig_cache &c, const tig_cache_attend &p)
{
    AttendPlan L = {};
    const int group = p.q_heads / c.heads, es = dtype_bytes(c.dtype), kt = es == 4 ? 16 : 32;
    // (four to a head: 300 us for 4000 histories, 280 on the matrix units; two of 256 columns: no registers)
    L.few = es != 4 ? 0 : group == 1 ? 1 : group == 2 && c.head_dim <= 128 ? 2 : 0;
    L.qt = group > 16 && c.head_dim <= 128 ? 2 : 1;
    L.rows = std::min(group, 16 * L.qt);
    L.blocks = (group + 16 * L.qt - 1) / (16 * L.qt);
    L.rec = (int64_t)L.rows * (c.head_dim + 2);
    const int64_t cap = p.window > 0 ? std::min<int64_t>(p.window, (int64_t)c.max_pages * c.page_size) : (int64_t)c.max_pages * c.page_size;
    const int64_t units = (int64_t)c.heads * L.blocks, tiles = cap / kt + 2, all = p.seqs * units * (tiles + kUnitCost);
    // A workgroup for each unit and one launch where there are few tiles for its wavefronts.  8 heads of 128 columns in bf16: 300 rows 10.4 us
    // this way, 14.5 the other one, 1000 rows 16.7 and 15.1, 4000 rows 42 and 17.5; 64 such units of 1000 rows 17.8 and 19.7, 256 of them 26 and 34.5.
    // (The table's width stands for the lengths here and below, which only the device knows: a table as wide as the longest sequence there may
    // be has short ones worked on the way of long ones.)
    L.solo = p.seqs * units <= 256 && tiles <= (p.seqs * units >= 64 ? 34 : 14);
    if (L.solo) {
        L.wgs = (int)(p.seqs * units), L.together = 1;
        return L;
    }
    // Wavefronts that go through the same rows together where these lie side by side and share lines of 128 bytes (4000 histories of two heads of
    // 200 bytes 319 us each by itself, 236 together), or where few long sequences are all there is (4 x 131071 rows of 8 x 256 bytes 404 and
    // 390; 77 sequences of 16 x 128 bytes 130 and 133).
    const bool side_by_side = c.heads > 1 && c.head_stride < c.token_stride;
    L.together = !side_by_side || all < 16384 ? 1 : c.head_stride * es % 128 != 0 ? (units >= 3 ? 4 : 2) : p.seqs * units <= 128 ? 2 : 1;
    const int64_t waves = (all + L.together - 1) / L.together;
    // A workgroup for each compute unit, one wavefront for each SIMD, fills the memory (4 x 131071 rows: 390 us, with two or four of them 402 and
    // 421); two where there are many units of few tiles, whose ends nothing runs beside (4000 histories of up to 100 rows 51 and 44 us, of up to
    // 3000 236 and 256; 600 sequences of up to 500 rows of 8 x 256 bytes 132 and 134).
    const int wanted = p.seqs * units >= 2048 * L.together && tiles <= 34 && c.head_dim <= 128 && L.qt == 1 ? 512 : 256;
    L.wgs = (int)std::min<int64_t>(wanted, (waves + kAttendWaves / L.together - 1) / (kAttendWaves / L.together));
    const int64_t most = (cap + kt - 1) / kt + (p.window > 0 && cap == p.window ? 1 : 0);  // tiles of a unit
    L.joins = L.wgs > 1 && most > kNeverShared;
    L.tails = ((int64_t)L.wgs * L.together * 2 * L.rec * 4 + 255) / 256 * 256;
    L.bytes = (size_t)(L.tails + ((int64_t)L.wgs * L.together * sizeof(Tail) + 255) / 256 * 256);
    return L;
}

template <class A, int WAVES, bool SOLO>
hipError_t launch_attend_main(const AttendArgs &a, const AttendPlan &L, hipStream_t s)
{
    const int lds = (int)(WAVES * 2 * L.rec * 4);
    auto *const kernel = k_cache_attend<A, WAVES, SOLO>;
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess)
            return e;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)L.wgs), dim3(64 * WAVES), (unsigned)lds, s, a);
    return hipGetLastError();
}
// solo_waves: wavefronts of a workgroup for each unit, as many as have the registers
template <class A, int SOLO_WAVES>
hipError_t launch_attend(const AttendArgs &a, const AttendPlan &L, hipStream_t s)
{
    if (L.solo)
        return launch_attend_main<A, SOLO_WAVES, true>(a, L, s);
    hipError_t e = launch_attend_main<A, kAttendWaves, false>(a, L, s);
    if (e == hipSuccess && L.joins) {
        const int lines = L.wgs * L.together;
        hipLaunchKernelGGL((k_cache_attend_join<typename A::Type>), dim3((unsigned)((lines + 3) / 4), (unsigned)L.rows), dim3(256), 0, s, a, lines);
        e = hipGetLastError();
    }
    return e;
}
template <typename T, int DP, bool PAGED>
hipError_t launch_attend_dim(const AttendArgs &a, const AttendPlan &L, hipStream_t s)
{
    if constexpr (sizeof(T) == 4) {
        if (L.few == 1)
            return launch_attend<AttendFew<DP, 1, PAGED>, (DP <= 128 ? 8 : 4)>(a, L, s);
        if constexpr (DP <= 128)
            if (L.few == 2)
                return launch_attend<AttendFew<DP, 2, PAGED>, 8>(a, L, s);
    }
    if constexpr (DP <= 128)
        if (L.qt == 2)
            return launch_attend<Attend<T, DP, 2, PAGED>, 4>(a, L, s);
    return launch_attend<Attend<T, DP, 1, PAGED>, (DP <= 128 ? 8 : 4)>(a, L, s);
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
    if (p->seqs > 0 && rows_meet(p->seqs, p->o_seq, p->q_heads, p->o_head, c->head_dim))
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
    if (L.bytes > 0 && (!workspace || ((uintptr_t)workspace & 255)))
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
    a.q_heads = p->q_heads, a.group = p->q_heads / cache->heads, a.blocks = L.blocks, a.rows = L.rows, a.window = p->window, a.together = L.together;
    a.scale = p->scale;
    a.factor = std::max(std::fabs(p->scale) * 1.44269504f, FLT_MIN);  // (not zero: a masked score times it has to stay -infinity)
    a.flip = p->scale < 0.0f ? (es == 4 ? 0x80000000u : 0x80008000u) : 0u;
    a.part = (float *)workspace, a.tails = (Tail *)((char *)workspace + L.tails), a.rec = L.rec;
    const hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = with_dtype(cache->dtype, [&](auto t) {
        using T = decltype(t);
        const int d = cache->head_dim;
        if (cache->page_size % 16 == 0)
            return d <= 64 ? launch_attend_dim<T, 64, true>(a, L, s) : d <= 128 ? launch_attend_dim<T, 128, true>(a, L, s) : launch_attend_dim<T, 256, true>(a, L, s);
        return d <= 64 ? launch_attend_dim<T, 64, false>(a, L, s) : d <= 128 ? launch_attend_dim<T, 128, false>(a, L, s) : launch_attend_dim<T, 256, false>(a, L, s);
    });
    return e == hipSuccess ? TIG_OK : fail_global("tig_cache_attend_run", e);
}
