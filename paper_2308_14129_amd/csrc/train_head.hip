// Ranking head of a training step (include/tig.h, tig_train_head): the sources' embeddings through a dense layer with a residual
// and a softmax cross entropy over the candidate nodes, and the way back.  The layer, the loss and their gradients are the
// library's own operators (linear.hip, softmax_ce.hip); here are the rows' way into and out of them.
#include <cmath>
#include <cstring>

#include "train.h"

namespace tig {

namespace {

inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

struct HeadLayout {
    float *P, *G;            // parameters and gradients: W, c, items, item_bias, each from a 256-byte boundary on
    size_t n;                // floats of either, gaps included
    size_t at[4], len[4];
    float *X, *H, *Z, *DH, *DX;  // [B x E]
    int32_t *labels;         // [B]
    double *demb;            // [2B x E]
    float *mean;
    void *opt_list;          // an optimiser's list of chunks
    void *ops;               // the operators' workspace
    size_t ops_bytes, bytes;
};

tig_linear head_linear(const Dims &d, const TrainHead &h, const HeadLayout &L, int64_t rows)
{
    tig_linear p;
    memset(&p, 0, sizeof(p));
    const int64_t E = d.E;
    p.struct_size = sizeof(p);
    p.dtype = TIG_F32, p.activation = h.activation;
    p.rows = rows, p.in_dim = p.out_dim = E;
    p.x = p.residual = L.X, p.w = L.P + L.at[0], p.bias = L.P + L.at[1], p.y = L.H, p.z = L.Z;
    p.dy = L.DH, p.dx = L.DX, p.dw = L.G + L.at[0], p.dbias = L.G + L.at[1];
    p.ldx = p.ldw = p.ldr = p.ldy = p.ldz = p.lddy = p.lddx = p.lddw = E;
    return p;
}

tig_softmax_ce head_loss(const Dims &d, const TrainHead &h, const HeadLayout &L, int64_t rows)
{
    tig_softmax_ce p;
    memset(&p, 0, sizeof(p));
    p.struct_size = sizeof(p);
    p.dtype = TIG_F32;
    p.rows = rows, p.vocab = h.num_items, p.dim = d.E;
    p.x = L.H, p.w = L.P + L.at[2], p.bias = L.P + L.at[3], p.labels = L.labels;
    p.scale = h.weight;
    p.mean = L.mean;
    p.dx = L.DH, p.dw = L.G + L.at[2], p.dbias = L.G + L.at[3];
    p.ldx = p.ldw = p.lddx = p.lddw = d.E;
    return p;
}

HeadLayout head_layout(const Dims &d, const TrainHead &h)
{
    HeadLayout L;
    memset(&L, 0, sizeof(L));
    const size_t E = d.E, B = d.max_batch, V = (size_t)h.num_items;
    const size_t len[4] = {E * E, E, V * E, V};
    for (int i = 0; i < 4; ++i) {
        L.at[i] = L.n, L.len[i] = len[i];
        L.n += (len[i] + 63) / 64 * 64;
    }
    size_t off = 0;
    // (addresses from 256 on where there is no workspace yet: the operators ask for their alignment only)
    char *const base = h.ws ? (char *)h.ws : (char *)256;
    auto take = [&](size_t bytes) -> void * {
        void *const p = base + off;
        off += align_up(bytes);
        return p;
    };
    L.P = (float *)take(4 * L.n);
    L.G = (float *)take(4 * L.n);
    L.X = (float *)take(4 * B * E);
    L.H = (float *)take(4 * B * E);
    L.Z = (float *)take(4 * B * E);
    L.DH = (float *)take(4 * B * E);
    L.DX = (float *)take(4 * B * E);
    L.labels = (int32_t *)take(4 * B);
    L.demb = (double *)take(8 * 2 * B * E);
    L.mean = (float *)take(4);
    int64_t n[kMaxTrainTensors], model[22];
    train_counts(d, model);
    memcpy(n, model, sizeof(model));
    for (int i = 0; i < 4; ++i)
        n[22 + i] = (int64_t)len[i];
    L.opt_list = take(adamw_list_bytes(n, kMaxTrainTensors));
    L.ops_bytes = h.ops_bytes;
    L.ops = take(L.ops_bytes);
    L.bytes = off;
    return L;
}

// Workgroup r clears row r of the rows' gradients; the first `count` also gather a source's embedding and its label.
__global__ void __launch_bounds__(128) k_head_rows(StepArgs a, int E, int64_t first_node, int64_t num_items, float *X, int32_t *labels, double *demb)
{
    const int r = (int)blockIdx.x;
    for (int j = threadIdx.x; j < E; j += 128)
        demb[(size_t)r * E + j] = 0.0;
    if (r >= a.count)
        return;
    const int row = row_of_entry_tr(a.qs, 2 * r, 2 * a.count);
    for (int j = threadIdx.x; j < E; j += 128)
        X[(size_t)r * E + j] = a.emb_u[(size_t)row * E + j];
    if (threadIdx.x == 0) {
        const int64_t item = (int64_t)a.dst[a.first_eid + r] - first_node;
        labels[r] = item >= 0 && item < num_items ? (int32_t)item : -1;
    }
}

// Gradients of an event's source embedding, through the layer and past it, to its query row.  In double: events that share a row
// come in any order, and a sum in fp32 would show which.
__global__ void __launch_bounds__(128) k_head_back(StepArgs a, int E, const float *DX, const float *DH, double *demb)
{
    const int b = (int)blockIdx.x, row = row_of_entry_tr(a.qs, 2 * b, 2 * a.count);
    for (int j = threadIdx.x; j < E; j += 128)
        unsafeAtomicAdd(&demb[(size_t)row * E + j], (double)DX[(size_t)b * E + j] + (double)DH[(size_t)b * E + j]);
}

__global__ void __launch_bounds__(256) k_head_sgd(float *P, const float *G, size_t n, float lr)
{
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256)
        P[i] -= lr * G[i];
}

hipError_t of_status(int rc) { return rc == TIG_OK ? hipSuccess : hipErrorUnknown; }

}  // namespace

// The most that a batch of any size needs: a smaller one may need more than the largest (sums split over more ranges).
size_t train_head_ops_bytes(const Dims &d, const TrainHead &h)
{
    const HeadLayout L = head_layout(d, h);
    size_t most = 256;
    for (int64_t rows = 1; rows <= d.max_batch; ++rows) {
        const tig_linear p = head_linear(d, h, L, rows);
        const tig_softmax_ce q = head_loss(d, h, L, rows);
        size_t n[3] = {0, 0, 0};
        (void)tig_linear_workspace_bytes(&p, 0, &n[0]);
        (void)tig_linear_workspace_bytes(&p, 1, &n[1]);
        (void)tig_softmax_ce_workspace_bytes(&q, &n[2]);
        for (size_t x : n)
            most = x > most ? x : most;
    }
    return most;
}

size_t train_head_bytes(const Dims &d, const TrainHead &h) { return head_layout(d, h).bytes; }
void *train_head_opt_list(const Dims &d, const TrainHead &h) { return head_layout(d, h).opt_list; }

hipError_t train_head_attach(const Dims &d, const TrainHead &h, const tig_train_head &from, hipStream_t s)
{
    const HeadLayout L = head_layout(d, h);
    const float *const src[4] = {from.W, from.c, from.items, from.item_bias};
    hipError_t e = launch_fill_zero(L.P, 4 * L.n, s);
    if (e == hipSuccess)
        e = launch_fill_zero(L.G, 4 * L.n, s);
    for (int i = 0; i < 4 && e == hipSuccess; ++i)
        e = hipMemcpyAsync(L.P + L.at[i], src[i], 4 * L.len[i], hipMemcpyDefault, s);
    return e;
}

hipError_t train_head_copy_out(const Dims &d, const TrainHead &h, bool grads, const tig_train_head &to, hipStream_t s)
{
    const HeadLayout L = head_layout(d, h);
    const float *const dst[4] = {to.W, to.c, to.items, to.item_bias};
    hipError_t e = hipSuccess;
    for (int i = 0; i < 4 && e == hipSuccess; ++i)
        if (dst[i])
            e = hipMemcpyAsync((void *)dst[i], (grads ? L.G : L.P) + L.at[i], 4 * L.len[i], hipMemcpyDefault, s);
    return e;
}

int train_head_tensors(const Dims &d, const TrainHead &h, float weight_decay, tig_adamw_tensor *out)
{
    const HeadLayout L = head_layout(d, h);
    for (int i = 0; i < 4; ++i) {
        out[i] = tig_adamw_tensor{};
        out[i].param = L.P + L.at[i], out[i].grad = L.G + L.at[i];
        out[i].n = (int64_t)L.len[i];
        out[i].weight_decay = i % 2 == 0 ? weight_decay : 0.0f;
    }
    return 4;
}

hipError_t launch_train_head(const Dims &d, const StepArgs &a, const TrainHead &h, const double **demb, const float **mean, int *launches, hipStream_t s)
{
    const HeadLayout L = head_layout(d, h);
    hipLaunchKernelGGL(k_head_rows, dim3((unsigned)(2 * a.count)), dim3(128), 0, s, a, d.E, h.first_node, h.num_items, L.X, L.labels, L.demb);
    hipError_t e = hipGetLastError();
    const tig_linear p = head_linear(d, h, L, a.count);
    const tig_softmax_ce q = head_loss(d, h, L, a.count);
    if (e == hipSuccess)
        e = of_status(tig_linear_forward(&p, L.ops, L.ops_bytes, s));
    if (e == hipSuccess)
        e = of_status(tig_softmax_ce_run(&q, L.ops, L.ops_bytes, s));
    if (e == hipSuccess)
        e = of_status(tig_linear_backward(&p, L.ops, L.ops_bytes, s));
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(k_head_back, dim3((unsigned)a.count), dim3(128), 0, s, a, d.E, L.DX, L.DH, L.demb);
    *demb = L.demb;
    *mean = L.mean;
    *launches += 2;  // (the operators' own launches are not counted)
    return hipGetLastError();
}

hipError_t launch_train_head_sgd(const Dims &d, const TrainHead &h, float lr, int *launches, hipStream_t s)
{
    const HeadLayout L = head_layout(d, h);
    const size_t blocks = (L.n + 255) / 256;
    hipLaunchKernelGGL(k_head_sgd, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, L.P, L.G, L.n, lr);
    ++*launches;
    return hipGetLastError();
}

}  // namespace tig
