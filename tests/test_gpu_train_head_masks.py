"""The ranking head of a training step with masked candidates."""
import math

import numpy as np
import pytest
import torch

import tig_synth as S
from oracle import tig_oracle as O
from tests import test_gpu_train_head as H
from tests.test_gpu_parity import Bundle, make_ctx

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(300)]


@pytest.fixture(scope="module")
def c1():
    return Bundle(S.WORKLOADS["c1_tiny"])


@pytest.mark.parametrize("order,activation", [("deferred", "silu"), ("update_first", "gelu")])
def test_candidates_that_are_nobodys_label(c1, order, activation, monkeypatch):
    """Finite losses: half of the candidates that no event of the batches turns to are masked."""
    g, plain = c1.g, H.make_head

    def masked_head(E, items, seed=0, masked=0):
        h = plain(E, items, seed)
        free = np.setdiff1d(np.arange(items), g.dst[6000:6400].astype(np.int64) - 3)
        assert len(free) > 20
        h["item_bias"][free[::2]] = -np.inf
        return h

    monkeypatch.setattr(H, "make_head", masked_head)
    H.run_head(c1, [(6000, 200), (6200, 200)], order, activation, 0.5, 3, 501, lr=0.01)


@pytest.mark.parametrize("order", ["deferred", "update_first"])
def test_labels_among_masked_candidates(c1, order):
    """An infinite loss; the gradients are those of the probabilities that are left, less the label's own."""
    H.run_head(c1, [(6000, 200), (6200, 130)], order, "gelu", 0.5, 0, c1.g.num_nodes, masked=c1.g.num_nodes // 2, lr=0.01)


def test_the_loss_is_infinite_where_a_label_is_masked(c1):
    w, g = c1.w, c1.g
    first, count = 6000, 100
    for masked_label in (False, True):
        head = H.make_head(w.emb_dim, g.num_nodes)
        labels = g.dst[first : first + count].astype(np.int64)
        if masked_label:
            head["item_bias"][labels[17]] = -np.inf
        ctx = make_ctx(w, g, c1.W, "fp32", count)
        ctx.train_attach(c1.W)
        ctx.train_head_attach(head, 0)
        st = O.OracleState(*S.make_warm_state(w, g, first))
        ctx.state_import(st.mem, st.last_update)
        loss = ctx.train_step(first, count, torch.from_numpy(S.make_negatives(w, g, first, count)).to("cuda:0"), ctx.alloc_outputs(count), 0.0)
        assert math.isinf(float(loss)) == masked_label
        assert all(np.isfinite(v).all() for v in {**ctx.train_get("grads"), **ctx.train_head_get("grads")}.values())
        ctx.close()
