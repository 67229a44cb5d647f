// One AdamW step over many tensors (include/tig.h, tig_adamw_*).  gfx950.
//
// The tensors are cut into chunks of 4096 elements, one workgroup each, listed once in the workspace: one launch whatever their
// number.  Bound by memory: every element's parameter and states are read and written once, its gradient read once, and once
// more where the norm is wanted.
//   k_adamw_norm    a chunk's sum of squares, in double
//   k_adamw_begin   joins them; the step's numbers (clip coefficient, bias corrections), the counter
//   k_adamw_update  the step
// 8-bit states: a wavefront takes 256 elements, four per lane, the block that shares a power of two: scales are exact, and
// values that do not change keep their code whatever the rest of their block does.
#include <cmath>
#include <cstring>
#include <new>

#include "act.h"
#include "gemm.h"

namespace tig {

namespace {

constexpr int kChunk = 4096, kStateBlock = 256, kAdamThreads = 256;

struct AdamTensor {
    void *param;
    const void *grad;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t n;
    int32_t dtype;
    int32_t wide;  // four elements at once, of every array
    float decay;
    int32_t pad;
};

struct AdamChunk {
    int32_t tensor, index;
};

// what k_adamw_begin leaves for the update
struct AdamNow {
    float c, step_size, root_scale, lr;
    uint32_t t;
    int32_t skip;
};

struct AdamParams {
    const AdamTensor *tensors;
    const AdamChunk *chunks;
    double *part;
    AdamNow *now;
    int64_t *step;
    int64_t n_chunks;
    double beta1, beta2, lr, grad_scale, max_norm;
    float b1, o1, b2, o2, eps;
    float *norm_out;
};

template <typename T>
__device__ inline double squares(const T *g, int64_t n, bool wide)
{
    double total = 0.0;
#pragma unroll
    for (int u = 0; u < kChunk / (4 * kAdamThreads); ++u) {
        const int64_t i = ((int64_t)u * kAdamThreads + threadIdx.x) * 4;
        if (i < n) {
            const floatx4 v = load_four(g + i, n - i < 4 ? (int)(n - i) : 4, wide);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                total += (double)v[e] * (double)v[e];
        }
    }
    return total;
}

__global__ void __launch_bounds__(kAdamThreads) k_adamw_norm(AdamParams p)
{
    __shared__ double part[kAdamThreads / kWave];
    const AdamChunk ch = p.chunks[blockIdx.x];
    const AdamTensor t = p.tensors[ch.tensor];
    const int64_t at = (int64_t)ch.index * kChunk, n = t.n - at < kChunk ? t.n - at : kChunk;
    double total = t.dtype == TIG_F32    ? squares((const float *)t.grad + at, n, t.wide)
                   : t.dtype == TIG_BF16 ? squares((const __bf16 *)t.grad + at, n, t.wide)
                                         : squares((const _Float16 *)t.grad + at, n, t.wide);
    for (int d = 32; d > 0; d >>= 1)
        total += __shfl_xor(total, d);
    if (lane_id() == 0)
        part[wave_id()] = total;
    __syncthreads();
    if (threadIdx.x == 0)
        p.part[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

__global__ void __launch_bounds__(1024) k_adamw_begin(AdamParams p)
{
    __shared__ double part[1024];
    double norm = 0.0;
    if (p.max_norm > 0.0) {
        double total = 0.0;
        for (int64_t i = threadIdx.x; i < p.n_chunks; i += 1024)
            total += p.part[i];
        part[threadIdx.x] = total;
        __syncthreads();
        for (int d = 512; d > 0; d >>= 1) {
            if ((int)threadIdx.x < d)
                part[threadIdx.x] += part[threadIdx.x + d];
            __syncthreads();
        }
        norm = fabs(p.grad_scale) * sqrt(part[0]);
    }
    if (threadIdx.x != 0)
        return;
    AdamNow now = {};
    now.skip = p.max_norm > 0.0 && !(norm < INFINITY);
    const int64_t t = *p.step + 1;
    double c = p.grad_scale;
    if (p.max_norm > 0.0 && norm > p.max_norm)
        c *= p.max_norm / norm;
    now.c = (float)c;
    now.lr = (float)p.lr;
    now.step_size = (float)(p.lr / (1.0 - pow(p.beta1, (double)t)));
    now.root_scale = (float)(1.0 / sqrt(1.0 - pow(p.beta2, (double)t)));
    now.t = (uint32_t)t;
    *p.now = now;
    if (!now.skip)
        *p.step = t;
    if (p.norm_out && p.max_norm > 0.0)
        *p.norm_out = (float)norm;
}

__device__ inline float wave_top(float v)
{
    for (int d = 32; d > 0; d >>= 1)
        v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// four values as e4m3 times the block's power of two; u: the thresholds
__device__ inline uint32_t to_8bit(const floatx4 &x, float top, const floatx4 &u, bool positive, float *scale)
{
    const int e0 = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) - 8 : 0;
    *scale = __builtin_amdgcn_ldexpf(1.0f, e0);
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float y = __builtin_amdgcn_ldexpf(fabsf(x[i]), -e0);
        int e = __builtin_amdgcn_frexp_expf(y);
        e = (e > -5 ? e : -5) - 4;
        float r = __builtin_amdgcn_ldexpf(floorf(__builtin_amdgcn_ldexpf(y, -e) + u[i]), e);
        if (positive)
            r = x[i] > 0.0f ? fmaxf(r, 0.001953125f) : r;
        else
            r = copysignf(r, x[i]);
        q[i] = r;
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
}
__device__ inline floatx4 from_8bit(uint32_t w, float scale)
{
    floatx4 v;
    v[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * scale;
    v[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * scale;
    v[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * scale;
    v[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * scale;
    return v;
}
__device__ inline uint32_t load_bytes(const uint8_t *p, int left, bool wide)
{
    if (left == 4 && wide)
        return *(const uint32_t *)p;
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        w |= e < left ? (uint32_t)p[e] << (8 * e) : 0u;
    return w;
}
__device__ inline void store_bytes(uint8_t *p, uint32_t w, int left, bool wide)
{
    if (left == 4 && wide) {
        *(uint32_t *)p = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left)
                p[e] = (uint8_t)(w >> (8 * e));
    }
}

// A wavefront's 256 elements from i on; products and sums in the order of the formulas, each rounded: a state's code does not
// depend on what the compiler joins.
template <typename T, int BITS>
__device__ inline void update_block(const AdamParams &p, const AdamTensor &t, const AdamNow &now, int64_t block, float keep)
{
#pragma clang fp contract(off)
    const int lane = lane_id();
    const int64_t i = block * kStateBlock + lane * 4;
    const int left = t.n - i < 4 ? (t.n > i ? (int)(t.n - i) : 0) : 4;
    const bool wide = t.wide != 0;
    const floatx4 g0 = load_four((const T *)t.grad + i, left, wide);
    floatx4 x = t.master ? load_four(t.master + i, left, wide) : load_four((const T *)t.param + i, left, wide);
    floatx4 m, v;
    if constexpr (BITS == 32) {
        m = load_four((const float *)t.m + i, left, wide);
        v = load_four((const float *)t.v + i, left, wide);
    } else {
        m = from_8bit(load_bytes((const uint8_t *)t.m + i, left, wide), t.m_scale[block]);
        v = from_8bit(load_bytes((const uint8_t *)t.v + i, left, wide), t.v_scale[block]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = v[e] * v[e];
    }
    floatx4 root;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float g = g0[e] * now.c;
        const float ma = m[e] * p.b1, mb = g * p.o1;
        m[e] = ma + mb;
        const float gg = g * g;
        const float va = v[e] * p.b2, vb = gg * p.o2;
        v[e] = va + vb;
        root[e] = sqrtf(v[e]);
        x[e] = x[e] * keep - now.step_size * (m[e] / (root[e] * now.root_scale + p.eps));
    }
    if (t.master)
        store_four(t.master + i, x, left, wide);
    store_four((T *)t.param + i, x, left, wide);
    if constexpr (BITS == 32) {
        store_four((float *)t.m + i, m, left, wide);
        store_four((float *)t.v + i, v, left, wide);
    } else {
        float top_m = 0.0f, top_r = 0.0f;
        floatx4 um, ur;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            top_m = fmaxf(top_m, e < left ? fabsf(m[e]) : 0.0f);
            top_r = fmaxf(top_r, e < left ? root[e] : 0.0f);
            const uint32_t h = (uint32_t)(lane * 4 + e) * 0x6A09E667u + now.t * 0x9E3779B9u;
            um[e] = (float)(h >> 8) * 0x1p-24f;
            ur[e] = (float)((h + 0x80000000u) >> 8) * 0x1p-24f;
        }
        float sm, sv;
        const uint32_t qm = to_8bit(m, wave_top(top_m), um, false, &sm), qr = to_8bit(root, wave_top(top_r), ur, true, &sv);
        store_bytes((uint8_t *)t.m + i, qm, left, wide);
        store_bytes((uint8_t *)t.v + i, qr, left, wide);
        if (lane == 0) {
            t.m_scale[block] = sm;
            t.v_scale[block] = sv;
        }
    }
}

template <typename T, int BITS>
__device__ inline void update_chunk(const AdamParams &p, const AdamTensor &t, const AdamNow &now, int64_t chunk)
{
    const float keep = 1.0f - now.lr * t.decay;
    const int64_t blocks = (t.n + kStateBlock - 1) / kStateBlock, first = chunk * (kChunk / kStateBlock);
#pragma unroll 2
    for (int u = 0; u < kChunk / kStateBlock / (kAdamThreads / kWave); ++u) {
        const int64_t b = first + u * (kAdamThreads / kWave) + wave_id_uniform();
        if (b < blocks)
            update_block<T, BITS>(p, t, now, b, keep);
    }
}

template <int BITS>
__global__ void __launch_bounds__(kAdamThreads) k_adamw_update(AdamParams p)
{
    const AdamNow now = *p.now;
    if (now.skip)
        return;
    const AdamChunk ch = p.chunks[blockIdx.x];
    const AdamTensor t = p.tensors[ch.tensor];
    if (t.dtype == TIG_F32)
        update_chunk<float, BITS>(p, t, now, ch.index);
    else if (t.dtype == TIG_BF16)
        update_chunk<__bf16, BITS>(p, t, now, ch.index);
    else
        update_chunk<_Float16, BITS>(p, t, now, ch.index);
}

inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct AdamLayout {
    int64_t n_chunks;
    size_t tensors, chunks, part, now, bytes;
};

AdamLayout adam_layout(const tig_adamw_tensor *t, int64_t n)
{
    AdamLayout L = {};
    for (int64_t i = 0; i < n; ++i)
        L.n_chunks += (t[i].n + kChunk - 1) / kChunk;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += align_up(bytes);
        return at;
    };
    L.tensors = take(sizeof(AdamTensor) * (size_t)n);
    L.chunks = take(sizeof(AdamChunk) * (size_t)L.n_chunks);
    L.part = take(sizeof(double) * (size_t)L.n_chunks);
    L.now = take(sizeof(AdamNow));
    L.bytes = off;
    return L;
}

int check_adamw(const tig_adamw_config *c, const tig_adamw_tensor *t, int64_t n)
{
    if (!c || c->struct_size != sizeof(tig_adamw_config))
        return fail_text(TIG_EINVAL, "tig_adamw: NULL configuration or wrong struct_size");
    if ((c->state_bits != 8 && c->state_bits != 32) || !(c->beta1 >= 0.0 && c->beta1 < 1.0) || !(c->beta2 >= 0.0 && c->beta2 < 1.0) ||
        !(c->eps > 0.0 && c->eps < 1e30) || !((float)c->eps > 0.0f))
        return fail_text(TIG_EINVAL, "tig_adamw: state_bits is 8 or 32, beta1 and beta2 in [0, 1), eps positive");
    if (!c->step || ((uintptr_t)c->step & 7))
        return fail_text(TIG_EINVAL, "tig_adamw: step is NULL or not 8-byte aligned");
    if (n < 0 || n > (1 << 20) || (n > 0 && !t))
        return fail_text(TIG_EINVAL, "tig_adamw: 0 to 2^20 tensors");
    int64_t chunks = 0;
    for (int64_t i = 0; i < n; ++i) {
        const tig_adamw_tensor &q = t[i];
        if (!dtype_ok(q.dtype) || q.n < 0 || q.n > ((int64_t)1 << 40) || !(q.weight_decay >= 0.0f && q.weight_decay < 1e30f))
            return fail_text(TIG_EINVAL, "tig_adamw: a tensor's dtype, size or weight_decay is out of range");
        if (q.n == 0)
            continue;
        if (!q.param || !q.grad || !q.m || !q.v)
            return fail_text(TIG_EINVAL, "tig_adamw: a tensor's param, grad, m or v is NULL");
        if (c->state_bits == 8 ? !q.m_scale || !q.v_scale : q.m_scale || q.v_scale)
            return fail_text(TIG_EINVAL, "tig_adamw: scales go with 8-bit states, and with these only");
        const uintptr_t es = (uintptr_t)dtype_bytes(q.dtype);
        if ((uintptr_t)q.param % es || (uintptr_t)q.grad % es || ((uintptr_t)q.master & 3) || ((uintptr_t)q.m_scale & 3) || ((uintptr_t)q.v_scale & 3) ||
            (c->state_bits == 32 && (((uintptr_t)q.m | (uintptr_t)q.v) & 3)))
            return fail_text(TIG_EINVAL, "tig_adamw: an address is not aligned to its element");
        chunks += (q.n + kChunk - 1) / kChunk;
        if (chunks > 0x7fffffff)
            return fail_text(TIG_EINVAL, "tig_adamw: more than 2^31 chunks of 4096 elements");
    }
    return TIG_OK;
}

}  // namespace

}  // namespace tig

using namespace tig;

struct tig_adamw {
    AdamParams p;
    int32_t bits;
};

int tig_adamw_workspace_bytes(const tig_adamw_config *cfg, const tig_adamw_tensor *tensors, int64_t n_tensors, size_t *bytes)
{
    const int rc = check_adamw(cfg, tensors, n_tensors);
    if (rc != TIG_OK)
        return rc;
    if (!bytes)
        return fail_text(TIG_EINVAL, "tig_adamw_workspace_bytes: bytes is NULL");
    *bytes = adam_layout(tensors, n_tensors).bytes;
    return TIG_OK;
}

int tig_adamw_create(const tig_adamw_config *cfg, const tig_adamw_tensor *tensors, int64_t n_tensors, void *workspace, size_t workspace_bytes,
                     void *hip_stream, tig_adamw **out)
{
    if (!out)
        return fail_text(TIG_EINVAL, "tig_adamw_create: out is NULL");
    *out = nullptr;
    const int rc = check_adamw(cfg, tensors, n_tensors);
    if (rc != TIG_OK)
        return rc;
    if (!workspace || ((uintptr_t)workspace & 255))
        return fail_text(TIG_EINVAL, "tig_adamw_create: workspace is NULL or not 256-byte aligned");
    const AdamLayout L = adam_layout(tensors, n_tensors);
    if (workspace_bytes < L.bytes)
        return fail_text(TIG_ENOSPACE, "tig_adamw_create: workspace too small");
    tig_adamw *const opt = new (std::nothrow) tig_adamw;
    char *const host = new (std::nothrow) char[L.part ? L.part : 1];  // tensors and chunks
    if (!opt || !host) {
        delete opt;
        delete[] host;
        return fail_text(TIG_ENOMEM, "tig_adamw_create: out of host memory");
    }
    memset(host, 0, L.part);
    AdamTensor *const dt = (AdamTensor *)(host + L.tensors);
    AdamChunk *ch = (AdamChunk *)(host + L.chunks);
    for (int64_t i = 0; i < n_tensors; ++i) {
        const tig_adamw_tensor &q = tensors[i];
        const int es = dtype_bytes(q.dtype), ss = cfg->state_bits == 32 ? 4 : 1;
        dt[i] = AdamTensor{q.param, q.grad, q.master, q.m, q.v, q.m_scale, q.v_scale, q.n, q.dtype, 0, q.weight_decay, 0};
        dt[i].wide = four_aligned(q.param, 4, es) && four_aligned(q.grad, 4, es) && four_aligned(q.master, 4, 4) && four_aligned(q.m, 4, ss) &&
                     four_aligned(q.v, 4, ss);
        for (int64_t c = 0; c < (q.n + kChunk - 1) / kChunk; ++c)
            *ch++ = AdamChunk{(int32_t)i, (int32_t)c};
    }
    hipStream_t s = (hipStream_t)hip_stream;
    hipError_t e = L.part ? hipMemcpyAsync(workspace, host, L.part, hipMemcpyHostToDevice, s) : hipSuccess;
    if (e == hipSuccess)
        e = hipStreamSynchronize(s);
    delete[] host;
    if (e != hipSuccess) {
        delete opt;
        return fail_global("tig_adamw_create", e);
    }
    AdamParams &p = opt->p;
    memset(&p, 0, sizeof(p));
    char *const ws = (char *)workspace;
    p.tensors = (const AdamTensor *)(ws + L.tensors);
    p.chunks = (const AdamChunk *)(ws + L.chunks);
    p.part = (double *)(ws + L.part);
    p.now = (AdamNow *)(ws + L.now);
    p.step = cfg->step;
    p.n_chunks = L.n_chunks;
    p.beta1 = cfg->beta1, p.beta2 = cfg->beta2;
    p.b1 = (float)cfg->beta1, p.o1 = (float)(1.0 - cfg->beta1), p.b2 = (float)cfg->beta2, p.o2 = (float)(1.0 - cfg->beta2);
    p.eps = (float)cfg->eps;
    opt->bits = cfg->state_bits;
    *out = opt;
    return TIG_OK;
}

int tig_adamw_step(tig_adamw *opt, double lr, double grad_scale, double max_norm, float *norm_out, void *hip_stream)
{
    if (!opt)
        return fail_text(TIG_EINVAL, "tig_adamw_step: NULL optimiser");
    if (!(lr >= 0.0 && lr < 1e30) || !(max_norm >= 0.0 && max_norm < 1e300) || !(std::fabs(grad_scale) < 1e30) || ((uintptr_t)norm_out & 3))
        return fail_text(TIG_EINVAL, "tig_adamw_step: lr and max_norm are finite and not negative, grad_scale is finite");
    AdamParams p = opt->p;
    p.lr = lr, p.grad_scale = grad_scale, p.max_norm = max_norm, p.norm_out = norm_out;
    hipStream_t s = (hipStream_t)hip_stream;
    const dim3 grid((unsigned)p.n_chunks);
    if (max_norm > 0.0 && p.n_chunks > 0)
        hipLaunchKernelGGL(k_adamw_norm, grid, dim3(kAdamThreads), 0, s, p);
    hipLaunchKernelGGL(k_adamw_begin, dim3(1), dim3(max_norm > 0.0 ? 1024 : 64), 0, s, p);
    if (p.n_chunks > 0) {
        if (opt->bits == 8)
            hipLaunchKernelGGL((k_adamw_update<8>), grid, dim3(kAdamThreads), 0, s, p);
        else
            hipLaunchKernelGGL((k_adamw_update<32>), grid, dim3(kAdamThreads), 0, s, p);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TIG_OK : fail_global("tig_adamw_step", e);
}

void tig_adamw_destroy(tig_adamw *opt) { delete opt; }
