"""The training step with a ranking head (dense layer with residual, softmax cross entropy over candidate nodes) and with
AdamW in place of SGD: losses and every gradient against the oracle, updates against their formulas in 64 bits."""
import ctypes
import math

import numpy as np
import pytest

import tig_synth as S
from oracle import tig_oracle as O
from oracle import train_oracle as T
from tests.parity import gate
from tests.test_gpu_parity import Bundle, make_ctx
from tests.test_gpu_train import GRAD_TOL, MAX_TIES, TIE_EPS, check_grads, compare_outputs_and_state, resolve_relu_ties

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(600)]

f32, f64 = np.float32, np.float64


@pytest.fixture(scope="module")
def c1():
    return Bundle(S.WORKLOADS["c1_tiny"])


def make_head(E, items, seed=0, masked=0):
    r = np.random.default_rng(seed)
    h = {"W": r.normal(0, E**-0.5, (E, E)).astype(f32), "c": r.uniform(-0.1, 0.1, E).astype(f32),
         "items": r.normal(0, 0.3, (items, E)).astype(f32), "item_bias": r.normal(0, 0.2, items).astype(f32)}
    h["item_bias"][r.permutation(items)[:masked]] = -np.inf
    return h


def act(z, name):
    if name == "gelu":
        phi = 0.5 * np.vectorize(math.erfc)(-z / math.sqrt(2))
        return z * phi, phi + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return z * s, s + z * s * (1 - s)
    if name == "relu":
        return np.maximum(z, 0), (z > 0).astype(f64)
    return z, np.ones_like(z)


def head_oracle(h, activation, labels, weight, keep):
    """The head's loss and gradient as train_oracle's `head`; the parameters' gradients go to `keep`."""
    p = {k: v.astype(f64) for k, v in h.items()}

    def run(emb):
        n = len(labels)
        e = emb[:n]
        z = e @ p["W"].T + p["c"]
        a, da = act(z, activation)
        hid = a + e
        logits = hid @ p["items"].T + p["item_bias"]
        lse = np.logaddexp.reduce(logits, axis=1)
        on = labels >= 0
        count = max(1, int(on.sum()))
        rows = np.flatnonzero(on)
        loss = float((lse[rows] - logits[rows, labels[rows]]).sum()) / count
        P = np.exp(logits - lse[:, None])
        P[rows, labels[rows]] -= 1
        P *= on[:, None] * weight / count
        dh = P @ p["items"]
        dz = dh * da
        keep.update(items=P.T @ hid, item_bias=P.sum(0), W=dz.T @ e, c=dz.sum(0))
        d = np.zeros_like(emb)
        d[:n] = dh + dz @ p["W"]
        return weight * loss, d

    return run


def run_head(bundle, batches, order, activation, weight, first_node, num_items, masked=0, lr=0.0):
    import torch
    w, g, ix = bundle.w, bundle.g, bundle.ix
    W = {k: v.copy() for k, v in bundle.W.items()}
    warm_at = batches[0][0]
    ctx = make_ctx(w, g, W, "fp32", max(c for _, c in batches), order)
    ctx.train_attach(W)
    head = make_head(w.emb_dim, num_items, masked=masked)
    ctx.train_head_attach(head, first_node, activation, weight)
    st = O.OracleState(*S.make_warm_state(w, g, warm_at))
    ctx.state_import(st.mem, st.last_update)
    for first, count in batches:
        print(f"[head {w.name} {order} {activation}] first_eid={first} count={count} lr={lr}", flush=True)
        neg = S.make_negatives(w, g, first, count)
        labels = g.dst[first : first + count].astype(np.int64) - first_node
        labels[(labels < 0) | (labels >= num_items)] = -1
        before, W0, keep = st.copy(), {k: v.copy() for k, v in W.items()}, {}
        args = (g.src, g.dst, g.ts, g.edge_feat, W, first, count, neg, w.num_neighbors, w.num_heads, lr)
        kw = dict(index=ix, deferred=order == "deferred", head=head_oracle(head, activation, labels, weight, keep))
        ref, loss, grads = T.train_step(st, *args, tie_eps=TIE_EPS, **kw)
        out = ctx.alloc_outputs(count)
        got_loss = ctx.train_step(first, count, torch.from_numpy(neg).to("cuda:0"), out, lr)
        torch.cuda.synchronize()
        compare_outputs_and_state(ctx, out, ref, st, 1e-4)
        assert float(got_loss.item()) == pytest.approx(loss, rel=2e-5) or math.isinf(loss)
        got = ctx.train_get("grads")
        try:
            check_grads(got, grads)
        except AssertionError:
            ties = ref.get("relu_ties", [])
            if not ties or len(ties) > MAX_TIES:
                raise

            def rerun(flips):
                W.update({k: v.copy() for k, v in W0.items()})
                return T.train_step(before.copy(), *args, relu_flip=flips, **kw)[2]
            check_grads(got, resolve_relu_ties(got, grads, ties, rerun))
        got_h = ctx.train_head_get("grads")
        for k in got_h:
            gate(got_h[k], keep[k], GRAD_TOL, f"head grad {k}")
        new_h, new_w = ctx.train_head_get("weights"), ctx.train_get("weights")
        for k in new_h:
            want = head[k].astype(f64) - lr * got_h[k].astype(f64)
            on = np.isfinite(head[k])
            # (one product and one difference in fp32, or both at once)
            assert (np.abs(new_h[k][on] - want[on]) <= 2.0**-23 * (np.abs(head[k][on]) + lr * np.abs(got_h[k][on]))).all()
            assert (new_h[k][~on] == head[k][~on]).all()
            head[k] = new_h[k]
        for k in T.PARAMS:
            gate(new_w[k].reshape(W[k].shape), W[k], 1e-5, f"weight {k}")
            W[k] = new_w[k].reshape(W[k].shape).copy()
    ctx.close()


@pytest.mark.parametrize("order", ["update_first", "deferred"])
@pytest.mark.parametrize("activation", ["gelu", "none"])
def test_head_gradients(c1, order, activation):
    # all nodes as candidates; ragged batches, one event
    run_head(c1, [(4000, 136), (4136, 200), (4336, 1), (4337, 64)], order, activation, 1.0, 0, c1.g.num_nodes)


def test_head_with_some_nodes_as_candidates_and_sgd(c1):
    # half of the destinations are no candidates, some candidates are masked (a label may be: the loss is then infinite)
    run_head(c1, [(6000, 200), (6200, 200)], "deferred", "silu", 0.5, 3, 501, lr=0.01)
    run_head(c1, [(6000, 100)], "update_first", "relu", 2.0, 2, 700, masked=0, lr=0.01)


def test_head_without_a_single_candidate_in_the_batch(c1):
    # the loss and the model's gradients are those of the step without a head, bit for bit where sums have one order
    import torch
    w, g = c1.w, c1.g
    first, count = 5000, 40
    unused = [n for n in range(g.num_nodes) if n not in set(g.dst[first : first + count].tolist())]
    node = next(n for n in unused if n + 1 in unused)
    neg = torch.from_numpy(S.make_negatives(w, g, first, count)).to("cuda:0")
    losses, grads = [], []
    for with_head in (False, True):
        ctx = make_ctx(w, g, c1.W, "fp32", count)
        ctx.train_attach(c1.W)
        if with_head:
            ctx.train_head_attach(make_head(w.emb_dim, 2), node)
        ctx.state_import(*S.make_warm_state(w, g, first))
        out = ctx.alloc_outputs(count)
        losses.append(float(ctx.train_step(first, count, neg, out, 0.0).item()))
        grads.append(ctx.train_get("grads"))
        if with_head:
            assert all(not v.any() for v in ctx.train_head_get("grads").values())
        ctx.close()
    assert losses[0] == losses[1]
    for k in T.PARAMS:
        gate(grads[1][k], grads[0][k].astype(f64), 1e-5, k) if k != "b_K" else None


DECAYED = {k for k in T.PARAMS if k[0] in "Ww" } | {"w_d2"}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("with_head,max_norm,decay", [(False, 0.0, 0.0), (True, 0.05, 0.1)])
def test_adamw_training_steps_follow_their_formula(c1, bits, with_head, max_norm, decay):
    """Each update from the gradients that the step itself reports; after it the model runs with the new weights."""
    import torch
    w, g = c1.w, c1.g
    ctx = make_ctx(w, g, c1.W, "fp32", 200, "deferred")
    ctx.train_attach(c1.W)
    if with_head:
        ctx.train_head_attach(make_head(w.emb_dim, 300), 10, weight=0.7)
    b1, b2, eps, lr = 0.9, 0.99, 1e-8, 1e-3
    ctx.train_adamw_attach((b1, b2), eps, decay, max_norm, bits)
    st = O.OracleState(*S.make_warm_state(w, g, 4000))
    ctx.state_import(st.mem, st.last_update)

    def params(what):
        p = dict(ctx.train_get(what))
        if with_head:
            p.update({"head " + k: v for k, v in ctx.train_head_get(what).items()})
        return {k: v.reshape(-1).astype(f64) for k, v in p.items()}

    old = params("weights")
    m, v = ({k: np.zeros_like(q) for k, q in old.items()} for _ in range(2))
    for t in range(1, 4 if bits == 32 else 2):  # (what 8 bits hold of a state is another test's matter: here the step that starts from zeros)
        first = 4000 + 200 * (t - 1)
        neg = S.make_negatives(w, g, first, 200)
        O.step(st, g.src, g.dst, g.ts, g.edge_feat, {k: old[k].reshape(c1.W[k].shape).astype(f32) for k in T.PARAMS}, first, 200, neg, w.num_neighbors,
               w.num_heads, index=c1.ix, deferred=True)
        out = ctx.alloc_outputs(200)
        ctx.train_step(first, 200, torch.from_numpy(neg).to("cuda:0"), out, lr)
        grad, new = params("grads"), params("weights")
        norm = math.sqrt(sum(float((q * q).sum()) for q in grad.values()))
        c = min(1.0, max_norm / norm) if max_norm else 1.0
        for k in old:
            d = decay if k in DECAYED or k in ("head W", "head items") else 0.0
            m[k] = b1 * m[k] + (1 - b1) * c * grad[k]
            v[k] = b2 * v[k] + (1 - b2) * (c * grad[k]) ** 2
            step = lr / (1 - b1**t) * m[k] / (np.sqrt(v[k] / (1 - b2**t)) + eps)
            want = old[k] * (1 - lr * d) - step
            tol = 2.0**-22 * (np.abs(old[k]) + 8 * np.abs(step) + 8 * lr)  # (a step is about lr; eight operations of a chain)
            assert (np.abs(new[k] - want) <= tol).all(), (k, t)
        if t == 1:
            assert any(np.abs(new[k] - old[k]).max() > 0.1 * lr for k in old)
        old = new
    # an ordinary step runs with the weights that the updates left
    first += 200
    neg = S.make_negatives(w, g, first, 200)
    W = {k: old[k].reshape(c1.W[k].shape).astype(f32) for k in T.PARAMS}
    ref = O.step(st, g.src, g.dst, g.ts, g.edge_feat, W, first, 200, neg, w.num_neighbors, w.num_heads, index=c1.ix, deferred=True)
    out = ctx.alloc_outputs(200)
    ctx.step(first, 200, torch.from_numpy(neg).to("cuda:0"), out)
    torch.cuda.synchronize()
    compare_outputs_and_state(ctx, out, ref, st, 1e-4)
    ctx.close()


def test_adamw_with_lr_zero_changes_nothing(c1):
    import torch
    w, g = c1.w, c1.g
    ctx = make_ctx(w, g, c1.W, "fp32", 50)
    ctx.train_attach(c1.W)
    ctx.train_head_attach(make_head(w.emb_dim, 20), 0)
    ctx.train_adamw_attach(max_norm=1.0)
    before, head = ctx.train_get("weights"), ctx.train_head_get("weights")
    out = ctx.alloc_outputs(50)
    ctx.train_step(4000, 50, torch.from_numpy(S.make_negatives(w, g, 4000, 50)).to("cuda:0"), out, 0.0)
    assert all(np.array_equal(before[k], v) for k, v in ctx.train_get("weights").items())
    assert all(np.array_equal(head[k], v) for k, v in ctx.train_head_get("weights").items())
    assert not ctx.adamw_ws[:8].any()  # the step counter
    ctx.close()


def test_head_and_optimiser_refusals(c1):
    import torch
    from paper_2308_14129_amd import tig
    w, g, E = c1.w, c1.g, c1.w.emb_dim
    ctx = make_ctx(w, g, c1.W, "fp32", 50)
    h = make_head(E, 30)

    def refused(call, status=tig.TIG_EINVAL):
        with pytest.raises(tig.TigError) as e:
            call()
        assert e.value.status == status

    refused(lambda: ctx.train_head_attach(h, 0))          # no training workspace
    refused(lambda: ctx.train_adamw_attach())
    ctx.train_attach(c1.W)
    refused(lambda: ctx.train_head_get("grads"))
    refused(lambda: ctx.train_head_attach(h, -1))
    refused(lambda: ctx.train_head_attach(h, g.num_nodes - 29))  # beyond the last node
    refused(lambda: ctx.train_head_attach(h, 0, weight=float("nan")))
    refused(lambda: ctx.train_head_attach(h, 0, "tanh"))
    refused(lambda: ctx.train_head_attach({**h, "W": h["W"][:, :5]}, 0))
    refused(lambda: ctx.train_head_attach({**h, "c": h["c"].astype(f64)}, 0))
    for bad in (dict(state_bits=16), dict(betas=(1.0, 0.9)), dict(eps=0.0), dict(weight_decay=-1.0), dict(max_norm=-1.0), dict(max_norm=float("inf"))):
        refused(lambda: ctx.train_adamw_attach(**bad))
    s = tig.tig_train_head(ctypes.sizeof(tig.tig_train_head), 2, 0, 30, 1.0, 0, *[h[k].ctypes.data for k in tig.HEAD_NAMES])
    n = ctypes.c_size_t(0)
    assert ctx.lib.tig_train_head_workspace_bytes(ctypes.byref(ctx.cfg), ctypes.byref(s), ctypes.byref(n)) == 0
    ws = torch.empty(n.value + 256, dtype=torch.uint8, device="cuda:0")
    assert ctx.lib.tig_train_head_attach(ctx.handle, ctypes.byref(s), ws.data_ptr(), n.value - 1) == tig.TIG_ENOSPACE
    assert ctx.lib.tig_train_head_attach(ctx.handle, ctypes.byref(s), ws.data_ptr() + 64, n.value) == tig.TIG_EINVAL
    s.W = None
    assert ctx.lib.tig_train_head_attach(ctx.handle, ctypes.byref(s), ws.data_ptr(), n.value) == tig.TIG_EINVAL
    ctx.train_adamw_attach()
    refused(lambda: ctx.train_head_attach(h, 0))          # the optimiser goes after the head
    ctx.train_attach(c1.W)                                # drops it
    ctx.train_head_attach(h, 0)
    ctx.train_adamw_attach(state_bits=8)
    ctx.train_adamw_attach(state_bits=32)
    ctx.close()
