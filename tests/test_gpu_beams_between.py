"""The selection's order between beams whose scores lie close to each other (ops.beam_select)."""
import pytest
import torch

from paper_2308_14129_amd import ops
from tests.paged import DEV, F64, TYPES, U, gen_of

pytestmark = [pytest.mark.gpu, pytest.mark.timeout(120)]


def beside_a_finished_beam(row, apart):
    """A finished beam, whose score is exact, `apart` above and below the best candidate of `row`: both in their places."""
    V = row.numel()
    x = torch.zeros(1, 2, V, device=DEV, dtype=row.dtype)
    x[0, 1] = row
    l = row.to(F64)
    best = float(l.max() - torch.logsumexp(l, 0))
    shift = torch.tensor(-best).float()  # brings the best candidate close to zero, where fp32 scores lie close to each other
    finished = torch.tensor([[True, False]], device=DEV)
    for side in (1, -1):
        scores = torch.stack([torch.tensor(best + float(shift.to(F64)) + side * apart, dtype=F64).float(), shift])[None].to(DEV)
        r = ops.beam_select(x, 1, scores, finished=finished, end=V - 1)
        assert r.parents.tolist() == [[0 if side > 0 else 1]], side
        assert int(r.tokens) == (V - 1 if side > 0 else int(torch.nonzero(l == l.max())[0]))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("seed", range(4))
def test_a_row_of_many_logits_beside_a_finished_beam(seed, dtype):
    """Of a million logits of a standard deviation of 1 about 370,000 carry the sum, each an exponential that is off by some 1.7e-7 (its
    argument and the difference before it, rounded; fp32's function), 3e-10 together; 244 sums of 4096 are off by some 4e-8 each, 3e-9
    together.  1.5e-8 is five times that.  A log2 e in fp32 alone leaves 1.3e-8 of the logits' distance from the largest one of their wavefront, all
    to one side: 2e-8 and more."""
    beside_a_finished_beam(torch.randn(1_000_003, device=DEV, generator=gen_of(100 + seed)).to(TYPES[dtype]), 1.5e-8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [1, 2, 50, 999, 32_000, 250_000])
def test_any_row_beside_a_finished_beam(V, dtype):
    """64 units of 2^-24 are what a log-sum of fp32 exponentials is off by at most, also where one distance makes up the sum."""
    gen = gen_of(V)
    for std in (0.0, 1.0, 4.0, 20.0):
        for peak in (0.0, 5.0, 12.43, 20.0):
            row = torch.randn(V, device=DEV, generator=gen) * std
            row[V // 3] += peak
            beside_a_finished_beam(row.to(TYPES[dtype]), 64 * U)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [100, 1000, 32_000, 250_000])
def test_beams_that_hold_one_row_in_several_orders(V, dtype):
    """Rotations of a row have one log-sum, up to the order of its sum: scores 1e-5 apart decide, scores that are alike leave it to the
    sums (the same from call to call), and each beam's own candidates are in order."""
    t, J, k = TYPES[dtype], 4, 16
    gen = gen_of(V)
    for row in (torch.randn(V, device=DEV, generator=gen), torch.rand(V, device=DEV, generator=gen).index_fill(0, torch.tensor([3], device=DEV), 5.0)):
        row = row.to(t)
        row[::7] = float("-inf")
        x = torch.stack([row, row.roll(V - 1), row.roll(V // 3), row.roll(V // 2 + 1)])[None].contiguous()
        alone = int((row == row.max()).sum()) == 1
        for scores in (torch.tensor([[0.0, 1e-5, -1e-5, 2e-5]], device=DEV), torch.zeros(1, J, device=DEV)):
            r = ops.beam_select(x, k, scores)
            value = torch.log_softmax(x[0].to(F64), -1) + scores[0].to(F64)[:, None]
            got = value[r.parents[0].long(), r.tokens[0].long()]
            want = value.flatten().sort(descending=True).values[:k]
            assert ((got - want).abs() <= 2 * 64 * U).all()
            assert ((r.scores[0].to(F64) - want).abs() <= U * want.abs() + 3 * 64 * U).all()
            for j in range(J):
                mine = [int(v) for p, v in zip(r.parents[0], r.tokens[0]) if int(p) == j]
                assert mine == sorted(mine, key=lambda v: (-float(x[0, j, v]), v))
            again = ops.beam_select(x, k, scores)
            assert torch.equal(again.parents, r.parents) and torch.equal(again.tokens, r.tokens)
            if scores.any() and alone and float(want[0] - want[4]) > 1e-4:
                assert r.parents[0, :4].tolist() == [3, 1, 0, 2]


def test_beams_alike_are_ties():
    """The same row in the same places has the same log-sum: the lowest beam first."""
    x = torch.randn(2, 1, 5000, device=DEV, generator=gen_of(8)).expand(2, 4, 5000)
    for logits in (x, x.contiguous()):
        r = ops.beam_select(logits, 8, torch.full((2, 4), -3.0, device=DEV))
        assert r.parents.tolist() == [[0, 1, 2, 3, 0, 1, 2, 3], [4, 5, 6, 7, 4, 5, 6, 7]]
        assert (r.tokens.view(2, 2, 4) == r.tokens.view(2, 2, 4)[..., :1]).all()
