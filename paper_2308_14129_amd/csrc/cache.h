// What the operators of a paged key-value cache share (include/tig.h, tig_cache).
#pragma once

#include <algorithm>
#include <initializer_list>

#include "act.h"
#include "gemm.h"

namespace tig {

// Division by the page size, one product: exact for numerators below 2^31.
struct PageDiv {
    uint32_t magic;
    int32_t shift, by;
    __device__ inline int quotient(int n) const { return (int)(((uint64_t)(uint32_t)n * magic) >> shift); }
};
// floor(2^(31 + l) / by) + 1 with 2^l >= by: its excess over 2^(31 + l) / by is at most 1, n < 2^31 of which are less than a 2^l-th, hence
// less than one by-th, of 2^(31 + l)
inline PageDiv page_div(int by)
{
    int l = 0;
    while ((1 << l) < by)
        ++l;
    return {(uint32_t)((((uint64_t)1 << (31 + l)) / (uint64_t)by) + 1), 31 + l, by};
}

// A cache and its sequences as kernels take them.
struct CacheView {
    char *k, *v;
    int64_t page_stride, token_stride, head_stride;  // bytes
    const int32_t *table, *lengths;
    int64_t ld_table;
    int32_t pages, page_size, heads, head_dim, max_pages;
    PageDiv div;

    __device__ inline int capacity() const { return max_pages * page_size; }
    __device__ inline int length(int64_t seq) const { return std::min(std::max(lengths[seq], 0), capacity()); }
    __device__ inline bool page_ok(int page) const { return (uint32_t)page < (uint32_t)pages; }
    __device__ inline int64_t offset(int page, int row, int head) const { return page * page_stride + row * token_stride + head * head_stride; }
};

inline CacheView cache_view(const tig_cache &c, const int32_t *table, int64_t ld_table, const int32_t *lengths)
{
    const int64_t es = dtype_bytes(c.dtype);
    return {(char *)c.k, (char *)c.v, c.page_stride * es, c.token_stride * es, c.head_stride * es, table, lengths, ld_table,
            (int32_t)c.pages, c.page_size, c.heads, c.head_dim, c.max_pages, page_div(c.page_size)};
}

int check_cache(const tig_cache *c);
// table and lengths of `seqs` sequences
int check_sequences(const tig_cache &c, int64_t seqs, const int32_t *table, int64_t ld, const int32_t *lengths);

// A tensor of up to three strided dimensions and adjacent columns, as rows that are one stride apart: its outer dimensions where they
// are one in memory, what lies within them as the columns.  (Views of one buffer that alternate stay apart that way: keys and
// values side by side, queries, keys and values of one product.)
struct Dim {
    int64_t n, stride;  // elements
};
Placed placed(const void *p, std::initializer_list<Dim> dims, int64_t cols, int elem);
inline Placed placed_keys(const tig_cache &c, const void *p)
{
    return placed(p, {{c.pages, c.page_stride}, {c.page_size, c.token_stride}, {c.heads, c.head_stride}}, c.head_dim, dtype_bytes(c.dtype));
}

// Whether two of the rows of `cols` elements at i * stride_a + j * stride_b, i < n_a and j < n_b, have an element in common.
bool rows_meet(int64_t n_a, int64_t stride_a, int64_t n_b, int64_t stride_b, int64_t cols);

// maximum / sum over a wavefront's lanes, for every lane
__device__ inline float wave_max_all(float v)
{
    v = row_max_all(v);
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// ... of the four lanes that share lane % 16
__device__ inline float groups_sum(float v)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
__device__ inline float wave_sum_all(float v) { return groups_sum(row_sum_all(v)); }

inline bool element_aligned(const void *p, int elem) { return (uintptr_t)p % (uintptr_t)elem == 0; }

// Bytes that are copied sixteen at a time wherever they start.
struct __attribute__((packed, aligned(2))) Sixteen {
    intx4 v;
};

// sixteen bytes of a row, the p-th or, where the row ends before, its last sixteen: then some are copied twice
__device__ inline int piece_start(int p, int row_bytes) { return std::min(16 * p, row_bytes - 16); }

}  // namespace tig
