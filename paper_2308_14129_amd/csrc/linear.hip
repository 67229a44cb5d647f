// Dense layer y = act(x W^T + b) + residual and its backward pass (include/tig.h, tig_linear_*).  gfx950.
//
//   up to 16 rows     k_linear_rows: the matrix is read once, straight into matrix-core operands
//   more rows         the tile product of gemm.h, bias, activation and residual in its epilogue
//   backward          k_linear_dz: dz = dy act'(z), and its column sums before it is rounded; then two tile products
// 8192 rows, 4096 -> 16384 in bf16 with gelu and residual: forward 1131 us, k_linear_dz 171 (4.7 TB/s), products 968 and 965.
// z is rounded to the layer's type when it is kept, and the slope is that of the rounded z.  dz is rounded too, to half a step of its
// own: it is a matrix operand of both products.  (With normal inputs dz's rounding adds as much error to the
// gradients as their own has, 1.7e-3 in bf16, and z's a third of that: 2.4e-3 together.)
#include <type_traits>

#include "act.h"
#include "gemm.h"

namespace tig {

namespace {

// Bias, activation, residual; z kept.
template <typename T, int ACT>
struct EpiLinear {
    static constexpr bool kWhole = false;
    const T *bias, *res;
    T *y, *z;
    int64_t ldr, ldy, ldz;
    struct Row {
        const T *res;
        T *y, *z;
    };
    __device__ inline Row row(int64_t m) const { return {res + m * ldr, y + m * ldy, z + m * ldz}; }
    template <bool FULL>
    __device__ inline floatx4 col(int64_t n, int left) const
    {
        return bias ? load_four(bias + n, FULL ? 4 : left) : floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    template <bool FULL>
    __device__ inline floatx4 load(const Row &r, int64_t n, int left) const
    {
        return res ? load_four(r.res + n, FULL ? 4 : left) : floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    template <bool FULL>
    __device__ inline void store(const Row &r, const floatx4 &b, const floatx4 &more, int64_t n, floatx4 v, int left) const
    {
        v += b;
        if (z)
            store_four(r.z + n, v, FULL ? 4 : left);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = activate<ACT>(v[e]);
        store_four(r.y + n, v + more, FULL ? 4 : left);
    }
};

// ------------------------------------------------------------------------------------------
// Few rows.  A workgroup takes sixteen columns of y for all rows; its wavefronts take turns along k, every lane loads 16 bytes
// of one row of W (and of x) as the matrix instructions want them, and the wavefronts' sums are added in LDS.
template <typename T>
__device__ inline intx4 operand_piece(const T *row, int64_t k, int64_t K)
{
    constexpr int per = Mat<T>::kPer16;
    struct __attribute__((packed, aligned(sizeof(T)))) Any {
        T v[per];
    };
    union {
        Any any;
        intx4 q;
    } u;
    if (k + per <= K) {
        u.any = *(const Any *)(row + k);
    } else {
#pragma unroll
        for (int e = 0; e < per; ++e)
            u.any.v[e] = k + e < K ? row[k + e] : (T)0.0f;
    }
    return u.q;
}

constexpr int kRowsWaves = 8;

// Up to sixteen rows: a workgroup takes sixteen columns, its wavefronts take turns along k, and both operands come straight from
// memory: a lane's sixteen bytes of a row are its part of an operand.  Bound by the matrix' bytes and, where it is small, by a
// launch and one chain of loads: one row, 1024 -> 4096 in bf16 3.4 us in a graph (2.5 TB/s), 16 rows, 4096 -> 16384 31 us (4.3 TB/s).
// The limit: 13 rows of 2000 -> 1333 in fp16 take 5.2 us here and 6.6 as tiles, 16 of 4096 -> 4096 in bf16 9.9 and 10.1, 48 of them
// (as three operands of sixteen) 18.1 and 12.1, 64 rows of 4096 -> 16384 73 and 33; in fp32 one row of 1024 -> 4096 4.8 and 9.3,
// 13 of 2000 -> 1333 6.9 and 11.1, 16 of 4096 -> 4096 17.4 and 23.6, 16 of 4096 -> 16384 62 and 80.  Four wavefronts instead of
// eight: the same within 2 % from 2048 to 32768 columns.
template <typename T, class Epi>
__global__ void __launch_bounds__(64 * kRowsWaves) k_linear_rows(const T *x, int64_t ldx, const T *w, int64_t ldw, int64_t M, int64_t N, int64_t K, Epi epi)
{
    constexpr int per = Mat<T>::kPer16, kBlock = 4 * per, kUnroll = 4, WAVES = kRowsWaves;
    __shared__ floatx4 red[WAVES][64];
    const int lane = lane_id(), wave = wave_id_uniform(), i16 = lane % 16, g = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * 16, n = n0 + i16 < N ? n0 + i16 : N - 1;
    const T *const wr = w + n * ldw + g * per, *const xr = x + (i16 < M ? i16 : M - 1) * ldx + g * per;
    floatx4 acc = {};
    const int64_t full = K / kBlock;  // blocks that are whole for every lane
    int64_t b = wave;
    for (; b + (kUnroll - 1) * WAVES < full; b += kUnroll * WAVES) {
        intx4 wv[kUnroll], xv[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int64_t k = (b + u * WAVES) * kBlock;
            wv[u] = operand_piece<T>(wr, k, k + per);
            xv[u] = operand_piece<T>(xr, k, k + per);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            mma16(acc, wv[u], xv[u], T());
    }
    for (; b * kBlock < K; b += WAVES) {
        const int64_t k = b * kBlock, left = K - g * per;
        mma16(acc, operand_piece<T>(wr, k, left), operand_piece<T>(xr, k, left), T());
    }
    red[wave][lane] = acc;
    __syncthreads();
    const int64_t c = n0 + 4 * g;
    if (wave == 0 && i16 < M && c < N) {
#pragma unroll
        for (int u = 1; u < WAVES; ++u)
            acc += red[u][lane];
        const int left = N - c < 4 ? (int)(N - c) : 4;
        const auto r = epi.row(i16);
        epi.template store<false>(r, epi.template col<false>(c, left), epi.template load<false>(r, c, left), c, acc, left);
    }
}

constexpr int64_t kFewRows = TIG_LINEAR_FEW_ROWS;
static_assert(kFewRows == 16, "one operand of rows");

template <typename T, class Epi>
hipError_t launch_linear_rows(const tig_linear &p, const Epi &epi, hipStream_t s)
{
    hipLaunchKernelGGL((k_linear_rows<T, Epi>), dim3((unsigned)((p.out_dim + 15) / 16)), dim3(64 * kRowsWaves), 0, s, (const T *)p.x, p.ldx, (const T *)p.w,
                       p.ldw, p.rows, p.out_dim, p.in_dim, epi);
    return hipGetLastError();
}

// ------------------------------------------------------------------------------------------
// dz = dy act'(z) for a block of rows and 64 pieces of 16 bytes (of dz) across, the wavefronts taking turns along the rows, and
// the block's column sums of dz before it is rounded.
constexpr int kDzWaves = 4;

template <typename T, int ACT>
__global__ void __launch_bounds__(64 * kDzWaves) k_linear_dz(const T *dy, int64_t lddy, const T *z, int64_t ldz, T *dz, int64_t lddz, float *sums,
                                                            int64_t lds, int64_t M, int64_t N, int64_t per, bool dy_ok, bool z_ok)
{
    constexpr int V = Mat<T>::kPer16 / 4, kDeep = 4;  // fours of a lane; rows on their way at a time
    __shared__ floatx4 part[kDzWaves][V][64];
    const int lane = lane_id(), wave = wave_id_uniform();
    const int64_t n0 = ((int64_t)blockIdx.x * 64 + lane) * (4 * V), m0 = (int64_t)blockIdx.y * per, m1 = m0 + per < M ? m0 + per : M;
    floatx4 total[V] = {};
    auto add = [&](int64_t m, floatx4 (&v)[V], const floatx4 (&q)[V]) {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            if constexpr (ACT != TIG_ACT_NONE)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[u][e] *= slope<ACT>(q[u][e]);
            total[u] += v[u];
        }
        if (dz)
            store_piece(dz + m * lddz + n0, v);
    };
    if (n0 + 4 * V <= N && dy_ok && z_ok) {
        int64_t m = m0 + wave;
        for (; m + (kDeep - 1) * kDzWaves < m1; m += kDeep * kDzWaves) {
            floatx4 v[kDeep][V], q[kDeep][V];
#pragma unroll
            for (int r = 0; r < kDeep; ++r) {
                load_piece(dy + (m + r * kDzWaves) * lddy + n0, v[r]);
                if constexpr (ACT != TIG_ACT_NONE)
                    load_piece(z + (m + r * kDzWaves) * ldz + n0, q[r]);
            }
#pragma unroll
            for (int r = 0; r < kDeep; ++r)
                add(m + r * kDzWaves, v[r], q[r]);
        }
        for (; m < m1; m += kDzWaves) {
            floatx4 v[V], q[V];
            load_piece(dy + m * lddy + n0, v);
            if constexpr (ACT != TIG_ACT_NONE)
                load_piece(z + m * ldz + n0, q);
            add(m, v, q);
        }
    } else if (n0 < (dz ? lddz : N)) {
        for (int64_t m = m0 + wave; m < m1; m += kDzWaves) {
            floatx4 v[V], q[V];
#pragma unroll
            for (int u = 0; u < V; ++u) {
                const int64_t n = n0 + 4 * u;
                const int left = N - n < 4 ? (N > n ? (int)(N - n) : 0) : 4;
                v[u] = load_four(dy + m * lddy + n, left);
                if constexpr (ACT != TIG_ACT_NONE)
                    q[u] = load_four(z + m * ldz + n, left);
            }
            add(m, v, q);
        }
    }
    if (!sums)
        return;
#pragma unroll
    for (int u = 0; u < V; ++u)
        part[wave][u][lane] = total[u];
    __syncthreads();
    for (int u = wave; u < V; u += kDzWaves) {
        const int64_t n = n0 + 4 * u;
        floatx4 v = part[0][u][lane];
#pragma unroll
        for (int w = 1; w < kDzWaves; ++w)
            v += part[w][u][lane];
        if (n < N)
            *(floatx4 *)(sums + (int64_t)blockIdx.y * lds + n) = v;
    }
}

// rows of a block: enough blocks to fill the chip, and no more than a grid's 65535
inline int64_t dz_rows(int64_t rows, int64_t cols, int per_lane)
{
    const int64_t across = (cols + 64 * per_lane - 1) / (64 * per_lane);
    int64_t per = 64;
    while (per > 16 && (rows + per - 1) / per * across < 1024)
        per /= 2;
    return (rows + per - 1) / per <= 65535 ? per : (rows + 65534) / 65535;
}

}  // namespace

// out[n] = scale * sum of the blocks' column sums, in double
template <typename T>
__global__ void __launch_bounds__(1024) k_join_sums(const float *sums, int64_t lds, int64_t blocks, int64_t N, T *out, const float *scale, float alpha)
{
    __shared__ double part[16][64];
    const int c = threadIdx.x % 64, w = threadIdx.x / 64;
    for (int64_t n0 = (int64_t)blockIdx.x * 64; n0 < N; n0 += (int64_t)gridDim.x * 64) {
        const int64_t n = n0 + c;
        double total = 0.0;
        if (n < N)
#pragma unroll 8
            for (int64_t b = w; b < blocks; b += 16)
                total += (double)sums[b * lds + n];
        part[w][c] = total;
        __syncthreads();
        if (w == 0 && n < N) {
            for (int k = 1; k < 16; ++k)
                total += part[k][c];
            out[n] = (T)(float)(total * (double)alpha * (scale ? (double)*scale : 1.0));
        }
        __syncthreads();
    }
}

template <typename T>
hipError_t launch_join_sums(const float *sums, int64_t lds, int64_t blocks, int64_t N, T *out, const float *scale, float alpha, hipStream_t s)
{
    const int64_t groups = (N + 63) / 64;
    hipLaunchKernelGGL((k_join_sums<T>), dim3((unsigned)(groups < 65536 ? groups : 65536)), dim3(1024), 0, s, sums, lds, blocks, N, out, scale, alpha);
    return hipGetLastError();
}
template hipError_t launch_join_sums<float>(const float *, int64_t, int64_t, int64_t, float *, const float *, float, hipStream_t);
template hipError_t launch_join_sums<__bf16>(const float *, int64_t, int64_t, int64_t, __bf16 *, const float *, float, hipStream_t);
template hipError_t launch_join_sums<_Float16>(const float *, int64_t, int64_t, int64_t, _Float16 *, const float *, float, hipStream_t);

namespace {

inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct LinearPlan {
    bool few;                      // forward: k_linear_rows
    GemmPlan y, dx, dw;
    bool pack_x, pack_w;           // operands whose rows are not 16-byte aligned
    bool store_dz;                 // backward: dz is written (else dy serves)
    int64_t ld_px, ld_pw, ld_dz, ld_sums, dz_per, sum_blocks;
    size_t px, pw, dz, sums, part;  // offsets into the workspace
    size_t bytes;
};

LinearPlan linear_plan(const tig_linear &p, bool backward)
{
    LinearPlan L = {};
    const int es = dtype_bytes(p.dtype);
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += align_up(bytes);
        return at;
    };
    L.ld_px = L.ld_pw = pack_ld(p.in_dim, es);
    if (p.rows == 0) {
        L.bytes = 0;
        return L;
    }
    if (!backward) {
        L.few = p.rows <= kFewRows;
        if (L.few)
            return L;
        L.pack_x = !gemm_fits(p.x, p.ldx, p.in_dim, es);
        L.pack_w = !gemm_fits(p.w, p.ldw, p.in_dim, es);
        L.y = gemm_plan(p.rows, p.out_dim, p.in_dim, es, true);
        L.part = take(L.y.part_bytes);
    } else {
        L.store_dz = (p.dx || p.dw) && (p.activation != TIG_ACT_NONE || !gemm_fits(p.dy, p.lddy, p.out_dim, es));
        L.pack_x = p.dw && !gemm_fits(p.x, p.ldx, p.in_dim, es);
        L.pack_w = p.dx && !gemm_fits(p.w, p.ldw, p.in_dim, es);
        L.dx = gemm_plan(p.rows, p.in_dim, p.out_dim, es, true);
        L.dw = gemm_plan(p.out_dim, p.in_dim, p.rows, es, true);
        size_t part = p.dx ? L.dx.part_bytes : 0;
        if (p.dw && L.dw.part_bytes > part)
            part = L.dw.part_bytes;
        L.part = take(part);
        L.ld_dz = pack_ld(p.out_dim, es);
        if (L.store_dz)
            L.dz = take((size_t)p.rows * L.ld_dz * es);
        L.dz_per = dz_rows(p.rows, L.ld_dz, 16 / es);
        L.sum_blocks = (p.rows + L.dz_per - 1) / L.dz_per;
        L.ld_sums = (p.out_dim + 3) / 4 * 4;
        if (p.dbias)
            L.sums = take((size_t)L.sum_blocks * L.ld_sums * 4);
    }
    if (L.pack_x)
        L.px = take((size_t)p.rows * L.ld_px * es);
    if (L.pack_w)
        L.pw = take((size_t)p.out_dim * L.ld_pw * es);
    L.bytes = off;
    return L;
}

int check_linear(const tig_linear *p, bool backward)
{
    if (!p || p->struct_size != sizeof(tig_linear))
        return fail_text(TIG_EINVAL, "tig_linear: NULL argument or wrong struct_size");
    if (!dtype_ok(p->dtype) || p->activation < TIG_ACT_NONE || p->activation > TIG_ACT_SILU || p->reserved != 0)
        return fail_text(TIG_EINVAL, "tig_linear: unknown dtype or activation, or reserved is not 0");
    if (p->rows < 0 || p->rows > (1 << 26) || p->in_dim < 1 || p->in_dim > kMaxDim || p->out_dim < 1 || p->out_dim > kMaxDim)
        return fail_text(TIG_EINVAL, "tig_linear: rows or dimensions out of range");
    auto ld_ok = [](int64_t ld, int64_t cols) { return ld >= cols && ld <= (1 << 22); };
    auto aligned = [&](const void *q) { return (uintptr_t)q % (uintptr_t)dtype_bytes(p->dtype) == 0; };
    const bool rows = p->rows > 0;
    if (!backward) {
        if (rows && (!p->x || !p->w || !p->y))
            return fail_text(TIG_EINVAL, "tig_linear_forward: x, w or y is NULL");
        if (!ld_ok(p->ldx, p->in_dim) || !ld_ok(p->ldw, p->in_dim) || !ld_ok(p->ldy, p->out_dim) || (p->residual && !ld_ok(p->ldr, p->out_dim)) ||
            (p->z && !ld_ok(p->ldz, p->out_dim)))
            return fail_text(TIG_EINVAL, "tig_linear_forward: a row stride is smaller than its row or above 2^22");
        if (!aligned(p->x) || !aligned(p->w) || !aligned(p->y) || !aligned(p->bias) || !aligned(p->residual) || !aligned(p->z))
            return fail_text(TIG_EINVAL, "tig_linear_forward: an address is not aligned to its element");
        return TIG_OK;
    }
    if (rows && (!p->dy || (p->dw && !p->x) || (p->dx && !p->w) || (p->activation != TIG_ACT_NONE && !p->z)))
        return fail_text(TIG_EINVAL, "tig_linear_backward: dy, z, or the x (w) that dw (dx) needs, is NULL");
    if (!ld_ok(p->lddy, p->out_dim) || (p->dw && (!ld_ok(p->ldx, p->in_dim) || !ld_ok(p->lddw, p->in_dim))) ||
        (p->dx && (!ld_ok(p->ldw, p->in_dim) || !ld_ok(p->lddx, p->in_dim))) || (p->activation != TIG_ACT_NONE && !ld_ok(p->ldz, p->out_dim)))
        return fail_text(TIG_EINVAL, "tig_linear_backward: a row stride is smaller than its row or above 2^22");
    if (!aligned(p->dy) || !aligned(p->x) || !aligned(p->w) || !aligned(p->z) || !aligned(p->dx) || !aligned(p->dw) || !aligned(p->dbias))
        return fail_text(TIG_EINVAL, "tig_linear_backward: an address is not aligned to its element");
    return TIG_OK;
}

// y may be residual itself; all else that is written keeps apart from what the call reads and writes.
int check_linear_apart(const tig_linear &p, bool backward)
{
    const int es = dtype_bytes(p.dtype);
    const int64_t r = p.rows, k = p.in_dim, n = p.out_dim;
    bool ok;
    if (!backward) {
        const bool in_place = p.y == p.residual && (p.ldy == p.ldr || r == 1);
        const Placed in[] = {{p.x, r, k, p.ldx, es}, {p.w, n, k, p.ldw, es}, {p.bias, 1, n, n, es}, {in_place ? nullptr : p.residual, r, n, p.ldr, es}};
        const Placed out[] = {{p.y, r, n, p.ldy, es}, {p.z, r, n, p.ldz, es}};
        ok = all_apart(in, out);
    } else {
        const Placed in[] = {{p.dy, r, n, p.lddy, es}, {p.dw ? p.x : nullptr, r, k, p.ldx, es}, {p.dx ? p.w : nullptr, n, k, p.ldw, es},
                             {p.activation != TIG_ACT_NONE ? p.z : nullptr, r, n, p.ldz, es}};
        const Placed out[] = {{p.dx, r, k, p.lddx, es}, {p.dw, n, k, p.lddw, es}, {p.dbias, 1, n, n, es}};
        ok = all_apart(in, out);
    }
    return ok ? TIG_OK : fail_text(TIG_EINVAL, "tig_linear: an output overlaps another tensor of the call");
}

int check_workspace(const void *workspace, size_t have, size_t need)
{
    if (need == 0)
        return TIG_OK;
    if (!workspace || ((uintptr_t)workspace & 255))
        return fail_text(TIG_EINVAL, "workspace is NULL or not 256-byte aligned");
    return have >= need ? TIG_OK : fail_text(TIG_ENOSPACE, "workspace too small");
}

template <typename T>
hipError_t forward(const tig_linear &p, const LinearPlan &L, char *ws, hipStream_t s)
{
    return with_activation(p.activation, [&](auto act) -> hipError_t {
        using Epi = EpiLinear<T, decltype(act)::value>;
        const int es = sizeof(T);
        const Epi epi = {(const T *)p.bias, (const T *)p.residual, (T *)p.y, (T *)p.z, p.ldr, p.ldy, p.ldz};
        if (L.few)
            return launch_linear_rows<T>(p, epi, s);
        const T *x = (const T *)p.x, *w = (const T *)p.w;
        int64_t ldx = p.ldx, ldw = p.ldw;
        hipError_t e = hipSuccess;
        if (L.pack_x) {
            e = launch_pack(x, ldx, ws + L.px, L.ld_px, p.rows, p.in_dim, es, s);
            x = (const T *)(ws + L.px), ldx = L.ld_px;
        }
        if (e == hipSuccess && L.pack_w) {
            e = launch_pack(w, ldw, ws + L.pw, L.ld_pw, p.out_dim, p.in_dim, es, s);
            w = (const T *)(ws + L.pw), ldw = L.ld_pw;
        }
        return e != hipSuccess ? e : launch_gemm<T, kRow, kRow>(L.y, x, ldx, w, ldw, p.rows, p.out_dim, p.in_dim, ws + L.part, epi, s);
    });
}

template <typename T>
hipError_t backward(const tig_linear &p, const LinearPlan &L, char *ws, hipStream_t s)
{
    const int es = sizeof(T);
    hipError_t e = hipSuccess;
    if (p.rows == 0) {
        if (p.dw)
            e = launch_zero_rows(p.dw, p.lddw, p.out_dim, p.in_dim, es, s);
        if (p.dbias && e == hipSuccess)
            e = launch_zero_rows(p.dbias, p.out_dim, 1, p.out_dim, es, s);
        return e;
    }
    const T *dz = (const T *)p.dy;
    int64_t lddz = p.lddy;
    if (L.store_dz || p.dbias) {
        T *const out = L.store_dz ? (T *)(ws + L.dz) : nullptr;
        float *const sums = p.dbias ? (float *)(ws + L.sums) : nullptr;
        const int64_t across = 64 * (16 / es);
        const dim3 grid((unsigned)((L.ld_dz + across - 1) / across), (unsigned)L.sum_blocks);
        with_activation(p.activation, [&](auto act) {
            hipLaunchKernelGGL((k_linear_dz<T, decltype(act)::value>), grid, dim3(64 * kDzWaves), 0, s, (const T *)p.dy, p.lddy, (const T *)p.z, p.ldz, out,
                               L.ld_dz, sums, L.ld_sums, p.rows, p.out_dim, L.dz_per, piece_aligned(p.dy, p.lddy, es), p.activation == TIG_ACT_NONE || piece_aligned(p.z, p.ldz, es));
            return 0;
        });
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
        if (out)
            dz = out, lddz = L.ld_dz;
        if (p.dbias && (e = launch_join_sums<T>(sums, L.ld_sums, L.sum_blocks, p.out_dim, (T *)p.dbias, nullptr, 1.0f, s)) != hipSuccess)
            return e;
    }
    if (p.dx) {
        const T *w = (const T *)p.w;
        int64_t ldw = p.ldw;
        if (L.pack_w) {
            e = launch_pack(w, ldw, ws + L.pw, L.ld_pw, p.out_dim, p.in_dim, es, s);
            w = (const T *)(ws + L.pw), ldw = L.ld_pw;
        }
        const EpiStore<T> epi = {(T *)p.dx, p.lddx, nullptr, 1.0f};
        if (e == hipSuccess)
            e = launch_gemm<T, kRow, kCol>(L.dx, dz, lddz, w, ldw, p.rows, p.in_dim, p.out_dim, ws + L.part, epi, s);
        if (e != hipSuccess)
            return e;
    }
    if (p.dw) {
        const T *x = (const T *)p.x;
        int64_t ldx = p.ldx;
        if (L.pack_x) {
            e = launch_pack(x, ldx, ws + L.px, L.ld_px, p.rows, p.in_dim, es, s);
            x = (const T *)(ws + L.px), ldx = L.ld_px;
        }
        const EpiStore<T> epi = {(T *)p.dw, p.lddw, nullptr, 1.0f};
        if (e == hipSuccess)
            e = launch_gemm<T, kCol, kCol>(L.dw, dz, lddz, x, ldx, p.out_dim, p.in_dim, p.rows, ws + L.part, epi, s);
    }
    return e;
}

}  // namespace

}  // namespace tig

using namespace tig;

int tig_linear_workspace_bytes(const tig_linear *p, int32_t backward, size_t *bytes)
{
    const int rc = check_linear(p, backward != 0);
    if (rc != TIG_OK)
        return rc;
    if (!bytes)
        return fail_text(TIG_EINVAL, "tig_linear_workspace_bytes: bytes is NULL");
    *bytes = linear_plan(*p, backward != 0).bytes;
    return TIG_OK;
}

int tig_linear_forward(const tig_linear *p, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_linear(p, false);
    if (rc != TIG_OK || p->rows == 0)
        return rc;
    const LinearPlan L = linear_plan(*p, false);
    if ((rc = check_workspace(workspace, workspace_bytes, L.bytes)) != TIG_OK || (rc = check_linear_apart(*p, false)) != TIG_OK)
        return rc;
    const hipError_t e = with_dtype(p->dtype, [&](auto t) { return forward<decltype(t)>(*p, L, (char *)workspace, (hipStream_t)hip_stream); });
    return e == hipSuccess ? TIG_OK : fail_global("tig_linear_forward", e);
}

int tig_linear_backward(const tig_linear *p, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = check_linear(p, true);
    if (rc != TIG_OK)
        return rc;
    const LinearPlan L = linear_plan(*p, true);
    if ((rc = check_workspace(workspace, workspace_bytes, L.bytes)) != TIG_OK || (rc = check_linear_apart(*p, true)) != TIG_OK)
        return rc;
    const hipError_t e = with_dtype(p->dtype, [&](auto t) { return backward<decltype(t)>(*p, L, (char *)workspace, (hipStream_t)hip_stream); });
    return e == hipSuccess ? TIG_OK : fail_global("tig_linear_backward", e);
}
