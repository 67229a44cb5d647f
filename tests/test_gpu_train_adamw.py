"""AdamW in the training step over several steps, and brought back from a copy of its workspace."""
import numpy as np
import pytest
import torch

import tig_synth as S
from oracle import train_oracle as T
from paper_2308_14129_amd import ops, tig
from tests.test_gpu_parity import Bundle, make_ctx
from tests.test_gpu_train_head import make_head

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]

B1, B2, EPS, LR = 0.9, 0.99, 1e-8, 1e-3
COUNT, FIRST = 150, 4000


@pytest.fixture(scope="module")
def c1():
    return Bundle(S.WORKLOADS["c1_tiny"])


def context(c1, weights, head, bits, max_norm):
    ctx = make_ctx(c1.w, c1.g, c1.W, "fp32", COUNT, "deferred")
    ctx.train_attach(weights)
    if head is not None:
        ctx.train_head_attach(head, 10, weight=0.7)
    ctx.train_adamw_attach((B1, B2), EPS, 0.1, max_norm, bits)
    return ctx


def train(c1, ctx, step):
    first = FIRST + COUNT * step
    neg = torch.from_numpy(S.make_negatives(c1.w, c1.g, first, COUNT)).to("cuda:0")
    ctx.train_step(first, COUNT, neg, ctx.alloc_outputs(COUNT), LR)
    torch.cuda.synchronize()


def flat(ctx, what, head):
    p = {k: v for k, v in ctx.train_get(what).items()}
    if head is not None:
        p.update({"head " + k: v for k, v in ctx.train_head_get(what).items()})
    return {k: v.reshape(-1).copy() for k, v in p.items()}


class Shadow:
    """ops.AdamW over copies of a context's parameters, fed with the gradients that its steps report."""

    def __init__(self, ctx, head, bits, max_norm):
        start = flat(ctx, "weights", head)
        self.names = list(T.PARAMS) + (["head W", "head c", "head items", "head item_bias"] if head is not None else [])
        assert set(self.names) == set(start)
        self.head, self.max_norm = head, max_norm
        self.p = [torch.from_numpy(start[k]).to("cuda:0") for k in self.names]
        self.g = [torch.zeros_like(q) for q in self.p]
        state = torch.float8_e4m3fn if bits == 8 else torch.float32
        m, v = ([torch.zeros(q.numel(), device="cuda:0").to(state) for q in self.p] for _ in range(2))
        ms, vs = ([torch.zeros(-(-q.numel() // 256), device="cuda:0") for q in self.p] if bits == 8 else None for _ in range(2))
        matrices = {k for k in self.names if k[0] in "Ww" or k in ("head W", "head items")}
        self.opt = ops.AdamW(self.p, self.g, m, v, torch.zeros(1, dtype=torch.int64, device="cuda:0"), m_scales=ms, v_scales=vs, betas=(B1, B2), eps=EPS,
                             weight_decay=[float(np.float32(0.1)) if k in matrices else 0.0 for k in self.names])

    def follow(self, ctx, what):
        """The step that ctx has just made: its weights are what this optimiser makes of its gradients, bit for bit."""
        grads, got = flat(ctx, "grads", self.head), flat(ctx, "weights", self.head)
        for q, k in zip(self.g, self.names):
            q.copy_(torch.from_numpy(grads[k]))
        self.opt.step(float(np.float32(LR)), max_norm=float(np.float32(self.max_norm)))
        for q, k in zip(self.p, self.names):
            assert np.array_equal(q.cpu().numpy(), got[k]), (what, k)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("with_head,max_norm", [(False, 0.0), (False, 0.5), (True, 0.0), (True, 0.05)])
def test_training_steps_are_the_optimisers_own(c1, bits, with_head, max_norm):
    head = make_head(c1.w.emb_dim, 300) if with_head else None
    ctx = context(c1, c1.W, head, bits, max_norm)
    ctx.state_import(*S.make_warm_state(c1.w, c1.g, FIRST))
    shadow = Shadow(ctx, head, bits, max_norm)
    for step in range(6):
        train(c1, ctx, step)
        shadow.follow(ctx, step)
    ctx.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("with_head", [False, True])
def test_optimiser_continues_in_another_context_from_a_copy_of_its_workspace(c1, bits, with_head):
    head = make_head(c1.w.emb_dim, 300) if with_head else None
    a = context(c1, c1.W, head, bits, 0.5)
    a.state_import(*S.make_warm_state(c1.w, c1.g, FIRST))
    shadow = Shadow(a, head, bits, 0.5)
    for step in range(3):
        train(c1, a, step)
        shadow.follow(a, step)
    saved, state = a.adamw_ws.cpu(), a.state_export()
    weights, params = a.train_get("weights"), a.train_head_get("weights") if with_head else None
    before = flat(a, "weights", head)
    # the first context lives on, so that nothing of the second one lies where the first one's does
    b = context(c1, weights, params, bits, 0.5)
    assert b.adamw_ws.numel() == saved.numel() and b.adamw_ws.data_ptr() != a.adamw_ws.data_ptr()
    b.adamw_ws.copy_(saved)
    torch.cuda.synchronize()
    b.state_import(*state)
    for step in range(3, 6):
        train(c1, b, step)
        assert int(b.adamw_ws[:8].view(torch.int64)) == step + 1
        shadow.follow(b, step)
    # nothing was written by way of the first context's addresses
    assert torch.equal(a.adamw_ws.cpu(), saved)
    for k, v in flat(a, "weights", head).items():
        assert np.array_equal(v, before[k]), k
    # and that one goes on as if nothing had been
    train(c1, a, 3)
    assert int(a.adamw_ws[:8].view(torch.int64)) == 4
    a.close()
    b.close()


def test_workspaces_are_the_contexts_streams(c1):
    """A context on a stream of its own, while the current stream still writes into memory that it has given back."""
    w, g = c1.w, c1.g
    cfg = tig.make_config(w.mem_dim, w.time_dim, w.feat_dim, w.emb_dim, w.num_neighbors, w.num_heads, COUNT, "fp32", "deferred")
    side = torch.cuda.Stream()
    ctx = tig.TigContext(cfg, g.num_nodes, g.src, g.dst, g.ts, g.edge_feat, c1.W, device="cuda:0", stream=side)
    head = make_head(w.emb_dim, 300)

    def attach():
        ctx.train_attach(c1.W)
        ctx.train_head_attach(head, 10)
        ctx.train_adamw_attach()
        return ctx.train_ws.numel(), ctx.head_ws.numel(), ctx.adamw_ws.numel()

    sizes = attach()
    torch.cuda.synchronize()
    held = [torch.empty(n, dtype=torch.uint8, device="cuda:0") for n in sizes]
    torch.cuda._sleep(400_000_000)
    for t in held:
        t.fill_(255)
    at = {t.data_ptr() for t in held}
    del held, t
    attach()
    assert not at & {ctx.train_ws.data_ptr(), ctx.head_ws.data_ptr(), ctx.adamw_ws.data_ptr()}
    torch.cuda.synchronize()
    for k, v in ctx.train_get("weights").items():
        assert np.array_equal(v.reshape(-1), c1.W[k].reshape(-1)), k
    for k, v in ctx.train_head_get("weights").items():
        assert np.array_equal(v, head[k]), k
    assert not ctx.adamw_ws.any()
    ctx.close()
