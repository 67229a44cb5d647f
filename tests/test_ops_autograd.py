"""The operators write no graph: tensors that want one are refused where graphs are recorded (no GPU needed)."""
import pytest
import torch

from paper_2308_14129_amd import ops, tig

X, W, B, LABELS = torch.zeros(4, 8), torch.zeros(6, 8), torch.zeros(6), torch.zeros(4, dtype=torch.int32)
Y, RS = torch.zeros(4, 6), torch.zeros(4)


def grad(t):
    return t.clone().requires_grad_()


CALLS = {
    "x": lambda: ops.linear(grad(X), W), "w": lambda: ops.linear(X, grad(W)), "bias": lambda: ops.linear(X, W, grad(B)),
    "residual": lambda: ops.linear(X, W, B, grad(Y)), "out": lambda: ops.linear(X, W, out=grad(Y)),
    "dy": lambda: ops.linear_backward(grad(Y), X, W), "x of the backward pass": lambda: ops.linear_backward(Y, grad(X), W),
    "z": lambda: ops.linear_backward(Y, X, W, grad(Y), "gelu"),
    "rows": lambda: ops.softmax_ce(grad(X), W, LABELS), "candidates": lambda: ops.softmax_ce(X, grad(W), LABELS),
    "candidates' bias": lambda: ops.softmax_ce(X, W, LABELS, grad(B)), "weights": lambda: ops.softmax_ce(X, W, LABELS, None, grad(RS)),
}


@pytest.mark.parametrize("which", CALLS)
def test_tensors_that_want_a_graph_are_refused(which):
    with pytest.raises(tig.TigError, match="no_grad") as e:
        CALLS[which]()
    assert e.value.status == tig.TIG_EINVAL
    with torch.no_grad(), pytest.raises(tig.TigError, match="not on a GPU"):  # (the next thing that is refused here)
        CALLS[which]()
