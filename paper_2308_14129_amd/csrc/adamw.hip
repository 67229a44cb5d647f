// One AdamW step over many tensors (include/tig.h, tig_adamw_*).  gfx950.
//
// The tensors are cut into chunks, one workgroup each, listed once in the workspace: one launch whatever their
// number.  Bound by memory: every element's parameter and states are read and written once, its gradient read once, and once
// more where the norm is wanted.
// 184 M elements with bf16 parameters and gradients, fp32 masters and states: the step 948 us (28 bytes an element, 5.4 TB/s), the
// norm 107 (3.4 TB/s); 219 M with 8-bit states 678 (16 bytes, 5.2 TB/s).
//   k_adamw_norm    sums of squares, in double (only with clipping)
//   k_adamw_begin   the step's numbers: clip coefficient, bias corrections, counter; few elements' update does that itself
//   k_adamw_update  the step
// 8-bit states: a wavefront takes the 256 elements that share a power of two, four per lane: scales are exact, and values that
// do not change keep their code whatever the rest of their block does.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "act.h"
#include "gemm.h"

namespace tig {

namespace {

constexpr int kStateBlock = 256, kAdamThreads = 256;
constexpr int kAtOnce = 4 * kAdamThreads;  // elements of a workgroup's round, four of a lane
// A chunk has four rounds, all of whose loads are on their way at once, or, where the tensors have up to 2^21 elements together,
// one: such a call is as long as a workgroup's chain of round trips (us for one and four rounds in fp32, without and with
// clipping: 2^18 elements 5.6 / 6.8 and 7.1 / 11.3, 2^21 10.2 / 14.1 and 10.7 / 15.3, 2^22 20.4 / 27.1 and 20.5 / 25.9, 2^24 66 / 100 and
// 69 / 80).
constexpr int kRoundsMany = 4, kRoundsFew = 1;
constexpr int64_t kFewElements = 1 << 21;
constexpr int kNormGroups = 8192;          // workgroups that form the norm, at most
constexpr int kFewGroups = 256;            // the same for few elements: every workgroup of the update adds their sums up

// A chunk of a tensor: where it lies.  (All of it in one record: from it to the data is one round trip.)
struct AdamChunk {
    void *param;
    const void *grad;
    float *master;
    void *m, *v;
    float *m_scale, *v_scale;
    int32_t n;
    int32_t dtype;
    float decay;
};

// the step's numbers
struct AdamNow {
    float c, step_size, root_scale, lr;
    int64_t t;
    int32_t skip;
};

struct AdamParams {
    const AdamChunk *chunks;
    double *part;       // [kNormGroups]
    AdamNow *now;
    int64_t *step;
    int64_t n_chunks;
    int n_parts;        // of `part`
    double beta1, beta2, lr, grad_scale, max_norm;
    float b1, o1, b2, o2, eps;
    float *norm_out;
};

// The step's numbers: what follows from the norm (0 without clipping) ...
__device__ inline void scale_by_norm(const AdamParams &p, double norm, AdamNow &now)
{
    now.skip = p.max_norm > 0.0 && !(norm < INFINITY);
    double c = p.grad_scale;
    if (p.max_norm > 0.0 && norm > p.max_norm)
        c *= p.max_norm / norm;
    now.c = (float)c;
}
// ... and from the number of the step.  (Half of a small update's time where each workgroup forms them after the norm.)
__device__ inline AdamNow numbers(const AdamParams &p, int64_t t)
{
    AdamNow now = {};
    now.lr = (float)p.lr;
    now.step_size = (float)(p.lr / (1.0 - pow(p.beta1, (double)t)));
    now.root_scale = (float)(1.0 / sqrt(1.0 - pow(p.beta2, (double)t)));
    now.t = t;
    return now;
}

template <int ROUNDS, typename T>
__device__ inline void load_grads(const T *g, int n, floatx4 (&v)[ROUNDS])
{
    if (n == ROUNDS * kAtOnce) {  // (uniform: a load in a lane's branch would be waited for at the branch's end)
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            v[r] = load_four(g + r * kAtOnce + (int)threadIdx.x * 4, 4);
    } else {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int i = r * kAtOnce + (int)threadIdx.x * 4;
            v[r] = load_four(g + i, n - i < 4 ? (n > i ? n - i : 0) : 4);
        }
    }
}

// the workgroup's sum of its threads' values, for every thread
__device__ inline double group_sum(double v)
{
    __shared__ double part[kAdamThreads / kWave];
    for (int d = 32; d > 0; d >>= 1)
        v += __shfl_xor(v, d);
    if (lane_id() == 0)
        part[wave_id()] = v;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// sums of squares in double, and the numbers that do not need them
template <int ROUNDS>
__global__ void __launch_bounds__(kAdamThreads) k_adamw_norm(AdamParams p)
{
    double total = 0.0;
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *p.now = numbers(p, *p.step + 1);
    // two chunks' loads on their way at a time
    for (int64_t c = blockIdx.x; c < p.n_chunks; c += 2 * (int64_t)gridDim.x) {
        const bool both = c + gridDim.x < p.n_chunks;  // (uniform)
        const AdamChunk ch[2] = {p.chunks[c], p.chunks[both ? c + gridDim.x : c]};
        floatx4 v[2][ROUNDS];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int n = k == 0 || both ? ch[k].n : 0;
            if (ch[k].dtype == TIG_F32)
                load_grads<ROUNDS>((const float *)ch[k].grad, n, v[k]);
            else if (ch[k].dtype == TIG_BF16)
                load_grads<ROUNDS>((const __bf16 *)ch[k].grad, n, v[k]);
            else
                load_grads<ROUNDS>((const _Float16 *)ch[k].grad, n, v[k]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    total += (double)v[k][r][e] * (double)v[k][r][e];
    }
    total = group_sum(total);
    if (threadIdx.x == 0)
        p.part[blockIdx.x] = total;
}

// the norm from the partial sums, always in the same order
__device__ inline double norm_of(const AdamParams &p)
{
    double total = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < p.n_parts; i += kAdamThreads)
        total += p.part[i];
    return fabs(p.grad_scale) * sqrt(group_sum(total));
}

// the step's numbers and the counter, ahead of an update of many chunks
__global__ void __launch_bounds__(kAdamThreads) k_adamw_begin(AdamParams p)
{
    const double norm = p.max_norm > 0.0 ? norm_of(p) : 0.0;
    if (threadIdx.x != 0)
        return;
    const int64_t t = *p.step + 1;
    AdamNow now = numbers(p, t);
    scale_by_norm(p, norm, now);
    *p.now = now;
    if (!now.skip)
        *p.step = t;
    if (p.norm_out && p.max_norm > 0.0)
        *p.norm_out = (float)norm;
}

// the largest over the wavefront
__device__ inline float wave_top(float v)
{
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x121, 0xf, 0xf, true)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x122, 0xf, 0xf, true)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x124, 0xf, 0xf, true)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, true)));
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// four values as e4m3 times their block's power of two; u: the thresholds
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
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
}
__device__ inline floatx4 from_8bit(uint32_t w, float scale)
{
    return floatx4{__builtin_amdgcn_cvt_f32_fp8((int)w, 0) * scale, __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * scale,
                   __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * scale, __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * scale};
}
struct __attribute__((packed)) FourBytes {
    uint32_t w;
};
__device__ inline uint32_t load_bytes(const uint8_t *p, int left)
{
    if (left == 4)
        return ((const FourBytes *)p)->w;
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left)
            w |= (uint32_t)p[e] << (8 * e);
    return w;
}
__device__ inline void store_bytes(uint8_t *p, uint32_t w, int left)
{
    if (left == 4) {
        ((FourBytes *)p)->w = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left)
                p[e] = (uint8_t)(w >> (8 * e));
    }
}

// A lane's fours of a chunk; numbers(): the step's, once the loads are on their way.  Products and sums in the order of the formulas, each rounded: a state's code does not depend
// on what the compiler joins.  A wavefront's four times 64 elements of a round are a block of 256.
template <typename T, int BITS, int ROUNDS, bool FULL, class F>
__device__ inline void update_chunk(const AdamParams &p, const AdamChunk &ch, const F &numbers)
{
#pragma clang fp contract(off)
    floatx4 g[ROUNDS], x[ROUNDS], m[ROUNDS], v[ROUNDS];
    uint32_t wm[ROUNDS], wv[ROUNDS];
    float sm[ROUNDS], sv[ROUNDS];
    const int i0 = (int)threadIdx.x * 4;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = i0 + r * kAtOnce, left = FULL || ch.n - i >= 4 ? 4 : (ch.n > i ? ch.n - i : 0);
        g[r] = load_four((const T *)ch.grad + i, left);
        x[r] = ch.master ? load_four(ch.master + i, left) : load_four((const T *)ch.param + i, left);
        if constexpr (BITS == 32) {
            m[r] = load_four((const float *)ch.m + i, left);
            v[r] = load_four((const float *)ch.v + i, left);
        } else {
            const int block = left > 0 ? i / kStateBlock : 0;
            wm[r] = load_bytes((const uint8_t *)ch.m + i, left);
            wv[r] = load_bytes((const uint8_t *)ch.v + i, left);
            sm[r] = ch.m_scale[block];
            sv[r] = ch.v_scale[block];
        }
    }
    const AdamNow now = numbers();
    if (now.skip)
        return;
    const float keep = 1.0f - now.lr * ch.decay;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = i0 + r * kAtOnce, left = FULL || ch.n - i >= 4 ? 4 : (ch.n > i ? ch.n - i : 0);
        if constexpr (BITS == 8) {
            m[r] = from_8bit(wm[r], sm[r]);
            v[r] = from_8bit(wv[r], sv[r]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[r][e] = v[r][e] * v[r][e];
        }
        floatx4 root;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float q = g[r][e] * now.c;
            const float ma = m[r][e] * p.b1, mb = q * p.o1;
            m[r][e] = ma + mb;
            const float qq = q * q;
            const float va = v[r][e] * p.b2, vb = qq * p.o2;
            v[r][e] = va + vb;
            root[e] = sqrtf(v[r][e]);
            x[r][e] = x[r][e] * keep - now.step_size * (m[r][e] / (root[e] * now.root_scale + p.eps));
        }
        if (ch.master)
            store_four(ch.master + i, x[r], left);
        store_four((T *)ch.param + i, x[r], left);
        if constexpr (BITS == 32) {
            store_four((float *)ch.m + i, m[r], left);
            store_four((float *)ch.v + i, v[r], left);
        } else {
            float top_m = 0.0f, top_r = 0.0f, a, b;
            floatx4 um, ur;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                top_m = fmaxf(top_m, e < left ? fabsf(m[r][e]) : 0.0f);
                top_r = fmaxf(top_r, e < left ? root[e] : 0.0f);
                const uint32_t h = (uint32_t)(i % kStateBlock + e) * 0x6A09E667u + (uint32_t)now.t * 0x9E3779B9u;
                um[e] = (float)(h >> 8) * 0x1p-24f;
                ur[e] = (float)((h + 0x80000000u) >> 8) * 0x1p-24f;
            }
            const uint32_t qm = to_8bit(m[r], wave_top(top_m), um, false, &a), qr = to_8bit(root, wave_top(top_r), ur, true, &b);
            store_bytes((uint8_t *)ch.m + i, qm, left);
            store_bytes((uint8_t *)ch.v + i, qr, left);
            if (left > 0 && lane_id() == 0) {
                ch.m_scale[i / kStateBlock] = a;
                ch.v_scale[i / kStateBlock] = b;
            }
        }
    }
}

// SELF: every workgroup forms the norm from the partial sums (few elements), the first one counts the step
template <int BITS, int ROUNDS, bool SELF>
__global__ void __launch_bounds__(kAdamThreads) k_adamw_update(AdamParams p)
{
    const AdamChunk ch = p.chunks[blockIdx.x];
    auto form = [&]() -> AdamNow {
        AdamNow now = *p.now;
        if constexpr (SELF) {
            const double norm = norm_of(p);
            scale_by_norm(p, norm, now);
            if (blockIdx.x == 0 && threadIdx.x == 0) {
                if (p.norm_out)
                    *p.norm_out = (float)norm;
                if (!now.skip)
                    *p.step = now.t;
            }
        }
        return now;
    };
    auto update = [&](auto type) {
        using T = decltype(type);
        if (ch.n == ROUNDS * kAtOnce)  // (uniform)
            update_chunk<T, BITS, ROUNDS, true>(p, ch, form);
        else
            update_chunk<T, BITS, ROUNDS, false>(p, ch, form);
    };
    if (ch.dtype == TIG_F32)
        update(float());
    else if (ch.dtype == TIG_BF16)
        update(__bf16());
    else
        update(_Float16());
}

inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct AdamLayout {
    int rounds;
    int64_t n_chunks;
    size_t chunks, part, now, bytes;
    int64_t chunk() const { return (int64_t)rounds * kAtOnce; }
};

AdamLayout adam_layout(const tig_adamw_tensor *t, int64_t n)
{
    AdamLayout L = {};
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i)
        total += t[i].n;
    L.rounds = total <= kFewElements ? kRoundsFew : kRoundsMany;
    for (int64_t i = 0; i < n; ++i)
        L.n_chunks += (t[i].n + L.chunk() - 1) / L.chunk();
    size_t off = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off += align_up(bytes);
        return at;
    };
    L.chunks = take(sizeof(AdamChunk) * (size_t)L.n_chunks);
    L.part = take(sizeof(double) * kNormGroups);  // (from here on nothing is laid out)
    L.now = take(sizeof(AdamNow));
    L.bytes = off;
    return L;
}

}  // namespace

size_t adamw_list_bytes(const int64_t *n, int n_tensors)
{
    tig_adamw_tensor t[kMaxTrainTensors] = {};
    for (int i = 0; i < n_tensors; ++i)
        t[i].n = n[i];
    return adam_layout(t, n_tensors).bytes;
}

namespace {

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
        chunks += (q.n + kRoundsMany * kAtOnce - 1) / (kRoundsMany * kAtOnce);
        if (chunks >= 1 << 24)  // (a launch's threads are counted in 32 bits)
            return fail_text(TIG_EINVAL, "tig_adamw: more than 2^24 chunks of 4096 elements");
    }
    return TIG_OK;
}

// Two workgroups must not step the same element, nor one step what another still reads: no array that the step writes overlaps
// another one.  (Gradients may overlap each other.)
int check_apart(const tig_adamw_config &c, const tig_adamw_tensor *t, int64_t n, const void *workspace, size_t workspace_bytes)
{
    struct Range {
        uintptr_t from, to;
        bool grad;
    };
    Range *const r = new (std::nothrow) Range[(size_t)(7 * n + 2)];
    if (!r)
        return fail_text(TIG_ENOMEM, "tig_adamw_create: out of host memory");
    int64_t k = 0;
    auto add = [&](const void *p, int64_t bytes, bool grad = false) {
        if (p && bytes > 0)
            r[k++] = Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, grad};
    };
    add(c.step, 8);
    add(workspace, (int64_t)workspace_bytes);
    for (int64_t i = 0; i < n; ++i) {
        const tig_adamw_tensor &q = t[i];
        const int64_t ss = c.state_bits == 32 ? 4 : 1, scales = (q.n + kStateBlock - 1) / kStateBlock * 4;
        add(q.param, q.n * dtype_bytes(q.dtype));
        add(q.grad, q.n * dtype_bytes(q.dtype), true);
        add(q.master, q.n * 4);
        add(q.m, q.n * ss);
        add(q.v, q.n * ss);
        add(q.m_scale, scales);
        add(q.v_scale, scales);
    }
    std::sort(r, r + k, [](const Range &a, const Range &b) { return a.from < b.from; });
    bool apart = true;
    uintptr_t read = 0, written = 0;  // ends of the ranges before
    for (int64_t i = 0; i < k; ++i) {
        apart = apart && written <= r[i].from && (r[i].grad || read <= r[i].from);
        uintptr_t &end = r[i].grad ? read : written;
        end = r[i].to > end ? r[i].to : end;
    }
    delete[] r;
    return apart ? TIG_OK : fail_text(TIG_EINVAL, "tig_adamw_create: an array that a step writes overlaps another one (a tensor given twice?)");
}

}  // namespace

}  // namespace tig

using namespace tig;

struct tig_adamw {
    AdamParams p;
    int32_t bits, rounds;
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
    int rc = check_adamw(cfg, tensors, n_tensors);
    if (rc != TIG_OK)
        return rc;
    if (!workspace || ((uintptr_t)workspace & 255))
        return fail_text(TIG_EINVAL, "tig_adamw_create: workspace is NULL or not 256-byte aligned");
    const AdamLayout L = adam_layout(tensors, n_tensors);
    if (workspace_bytes < L.bytes)
        return fail_text(TIG_ENOSPACE, "tig_adamw_create: workspace too small");
    if ((rc = check_apart(*cfg, tensors, n_tensors, workspace, L.bytes)) != TIG_OK)
        return rc;
    tig_adamw *const opt = new (std::nothrow) tig_adamw;
    char *const host = new (std::nothrow) char[L.part ? L.part : 1];  // the list of chunks
    if (!opt || !host) {
        delete opt;
        delete[] host;
        return fail_text(TIG_ENOMEM, "tig_adamw_create: out of host memory");
    }
    memset(host, 0, L.part);
    AdamChunk *ch = (AdamChunk *)(host + L.chunks);
    for (int64_t i = 0; i < n_tensors; ++i) {
        const tig_adamw_tensor &q = tensors[i];
        const int es = dtype_bytes(q.dtype), ss = cfg->state_bits == 32 ? 4 : 1;
        auto at = [](const void *x, int64_t bytes) { return x ? (void *)((char *)x + bytes) : nullptr; };
        for (int64_t c = 0; c < q.n; c += L.chunk())
            *ch++ = AdamChunk{at(q.param, c * es), at(q.grad, c * es), (float *)at(q.master, c * 4), at(q.m, c * ss), at(q.v, c * ss),
                              (float *)at(q.m_scale, c / kStateBlock * 4), (float *)at(q.v_scale, c / kStateBlock * 4),
                              (int32_t)(q.n - c < L.chunk() ? q.n - c : L.chunk()), q.dtype, q.weight_decay};
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
    p.chunks = (const AdamChunk *)(ws + L.chunks);
    p.part = (double *)(ws + L.part);
    p.now = (AdamNow *)(ws + L.now);
    p.step = cfg->step;
    p.n_chunks = L.n_chunks;
    p.beta1 = cfg->beta1, p.beta2 = cfg->beta2;
    p.b1 = (float)cfg->beta1, p.o1 = (float)(1.0 - cfg->beta1), p.b2 = (float)cfg->beta2, p.o2 = (float)(1.0 - cfg->beta2);
    p.eps = (float)cfg->eps;
    opt->bits = cfg->state_bits;
    opt->rounds = L.rounds;
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
    const bool clip = max_norm > 0.0, few = opt->rounds == kRoundsFew, self = clip && few && p.n_chunks > 0;
    const int64_t most = few ? kFewGroups : kNormGroups;
    p.n_parts = clip ? (int)(p.n_chunks < most ? p.n_chunks : most) : 0;
    const dim3 grid((unsigned)p.n_chunks), parts((unsigned)p.n_parts), threads(kAdamThreads);
    auto launch = [&](auto rounds) {
        constexpr int R = decltype(rounds)::value;
        if (p.n_parts > 0)
            hipLaunchKernelGGL((k_adamw_norm<R>), parts, threads, 0, s, p);
        if (!self)
            hipLaunchKernelGGL(k_adamw_begin, dim3(1), threads, 0, s, p);
        if (p.n_chunks == 0)
            return;
        auto *const update = opt->bits == 8 ? (self ? k_adamw_update<8, R, true> : k_adamw_update<8, R, false>)
                                            : (self ? k_adamw_update<32, R, true> : k_adamw_update<32, R, false>);
        hipLaunchKernelGGL(update, grid, threads, 0, s, p);
    };
    if (few)
        launch(std::integral_constant<int, kRoundsFew>());
    else
        launch(std::integral_constant<int, kRoundsMany>());
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? TIG_OK : fail_global("tig_adamw_step", e);
}

void tig_adamw_destroy(tig_adamw *opt) { delete opt; }
