"""What the paged cache and the selection over beams refuse, before anything reaches a GPU (no GPU needed)."""
import ctypes
import os
from ctypes import byref, c_size_t

import pytest
import torch

from paper_2308_14129_amd import ops, tig


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(tig.LIB_PATH):
        from paper_2308_14129_amd import build
        build.build()
    return ops._lib()


HOST = 0x10000  # addresses that are never read: every call here is refused first
MB = 1 << 20


def put(p, kw):
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def make_cache(**kw):
    """64 pages of 16 rows of 4 heads of 32 columns in bf16, row by row: 256 KiB each."""
    c = ops.tig_cache(ctypes.sizeof(ops.tig_cache), 1, 64, 16, 4, 32, 10, HOST, HOST + MB, 16 * 128, 128, 32)
    return put(c, kw)


def make_append(**kw):
    p = ops.tig_cache_append(ctypes.sizeof(ops.tig_cache_append), 32, 0, 0, 5, 5)
    for i, n in enumerate(("table", "lengths", "k", "v", "q", "q_out", "freq")):
        setattr(p, n, HOST + (8 + i) * MB)
    p.ld_table, p.q_heads = 10, 8
    p.k_token = p.v_token = 128
    p.q_token = p.qo_token = 256
    p.k_head = p.v_head = p.q_head = p.qo_head = 32
    return put(p, kw)


def make_attend(**kw):
    p = ops.tig_cache_attend(ctypes.sizeof(ops.tig_cache_attend), 0, 5, 8, 0.25)
    for i, n in enumerate(("table", "lengths", "q", "out", "lse")):
        setattr(p, n, HOST + (8 + i) * MB)
    p.ld_table, p.q_seq, p.q_head, p.o_seq, p.o_head = 10, 256, 32, 256, 32
    return put(p, kw)


def make_fork(**kw):
    p = ops.tig_cache_fork(ctypes.sizeof(ops.tig_cache_fork), 0, 5, 6)
    for i, n in enumerate(("table", "lengths", "parents", "spare", "table_out", "lengths_out")):
        setattr(p, n, HOST + (8 + i) * MB)
    p.ld_table = p.ld_out = 10
    return put(p, kw)


def make_select(**kw):
    p = ops.tig_beam_select(ctypes.sizeof(ops.tig_beam_select), 1, 3, 4, 4, 1000)
    for i, n in enumerate(("logits", "scores", "finished", "scores_out", "parents", "tokens", "finished_out")):
        setattr(p, n, HOST + i * MB)
    p.l_batch, p.l_beam, p.end = 4000, 1000, 2
    return put(p, kw)


CACHE = [
    dict(struct_size=8), dict(dtype=3), dict(dtype=-1), dict(pages=0), dict(pages=2**31), dict(page_size=0), dict(page_size=2**16 + 1), dict(heads=0),
    dict(heads=1025), dict(head_dim=7), dict(head_dim=257), dict(max_pages=0), dict(max_pages=2**24 + 1), dict(max_pages=2**24, page_size=128),
    dict(k=None), dict(v=None), dict(k=HOST + 1), dict(v=HOST + 1), dict(page_stride=-1), dict(token_stride=-1), dict(head_stride=-1),
    dict(page_stride=2**41), dict(head_stride=2**41), dict(head_stride=31), dict(token_stride=127), dict(page_stride=16 * 128 - 1), dict(page_stride=0),
    dict(token_stride=0), dict(token_stride=2**25 + 1, page_stride=2**30), dict(page_size=2**16, token_stride=128 * 128, page_stride=2**30, max_pages=1),
    dict(heads=1024, page_size=2**15, token_stride=32, head_stride=2**20, page_stride=2**30, max_pages=1)]
SEQS = [dict(seqs=-1), dict(seqs=2**20 + 1), dict(table=None), dict(lengths=None), dict(table=HOST + 2), dict(lengths=HOST + 1), dict(ld_table=9)]


@pytest.mark.parametrize("bad", CACHE, ids=str)
def test_cache(lib, bad):
    c, need = make_cache(**bad), c_size_t(0)
    assert lib.tig_cache_append_run(byref(c), byref(make_append()), None) == tig.TIG_EINVAL
    assert lib.tig_cache_attend_workspace_bytes(byref(c), byref(make_attend()), byref(need)) == tig.TIG_EINVAL
    assert lib.tig_cache_attend_run(byref(c), byref(make_attend()), HOST, 1 << 40, None) == tig.TIG_EINVAL
    assert lib.tig_cache_fork_run(byref(c), byref(make_fork()), None) == tig.TIG_EINVAL
    assert b"tig_cache:" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", SEQS + [
    dict(struct_size=8), dict(rotary=-2), dict(rotary=31), dict(rotary=34), dict(interleaved=2), dict(interleaved=-1), dict(reserved=1), dict(tokens=-1),
    dict(tokens=4), dict(tokens=2**23 + 1, starts=HOST), dict(position_type=3), dict(position_type=1), dict(positions=HOST), dict(freq=None), dict(rotary=0),
    dict(freq=HOST + 4), dict(position_type=1, positions=HOST + 4), dict(starts=HOST + 2), dict(q_heads=0), dict(q_heads=-1), dict(q_heads=2**14 + 1),
    dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(k=HOST + 1), dict(v=HOST + 1), dict(q=HOST + 1), dict(q_out=HOST + 1), dict(k_token=-1),
    dict(qo_head=2**33), dict(qo_token=31), dict(qo_head=31)], ids=str)
def test_append(lib, bad):
    c, p = make_cache(), make_append(**bad)
    assert lib.tig_cache_append_run(byref(c), byref(p), None) == tig.TIG_EINVAL
    assert b"cache" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", SEQS + [
    dict(struct_size=8), dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_heads=0), dict(q_heads=6), dict(q_heads=2**15), dict(q=None),
    dict(out=None), dict(q=HOST + 1), dict(out=HOST + 1), dict(lse=HOST + 2), dict(q_seq=-1), dict(o_head=2**33), dict(o_seq=31), dict(o_head=31),
    dict(o_seq=128)], ids=str)
def test_attend(lib, bad):
    c, p, need = make_cache(), make_attend(**bad), c_size_t(0)
    assert lib.tig_cache_attend_workspace_bytes(byref(c), byref(p), byref(need)) == tig.TIG_EINVAL
    assert lib.tig_cache_attend_run(byref(c), byref(p), HOST, 1 << 40, None) == tig.TIG_EINVAL
    assert b"cache" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", [{("rows_in" if k == "seqs" else k): v for k, v in b.items()} for b in SEQS] + [
    dict(struct_size=8), dict(reserved=1), dict(rows_out=-1), dict(rows_out=2**20 + 1), dict(parents=None), dict(spare=None), dict(table_out=None),
    dict(lengths_out=None), dict(parents=HOST + 2), dict(spare=HOST + 1), dict(table_out=HOST + 2), dict(lengths_out=HOST + 3), dict(ld_out=9)], ids=str)
def test_fork(lib, bad):
    c, p = make_cache(), make_fork(**bad)
    assert lib.tig_cache_fork_run(byref(c), byref(p), None) == tig.TIG_EINVAL
    assert b"cache" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", [
    dict(struct_size=8), dict(dtype=3), dict(reserved=1), dict(batch=-1), dict(batch=2**20 + 1), dict(beams=0), dict(beams=65), dict(k=0), dict(k=129), dict(vocab=0),
    dict(vocab=2**28 + 1), dict(beams=64, vocab=2**25), dict(batch=2**20, beams=32), dict(end=-2), dict(end=1000), dict(end=-1), dict(logits=None),
    dict(scores_out=None), dict(parents=None), dict(tokens=None), dict(logits=HOST + 1), dict(scores=HOST + 2), dict(tokens=HOST + 1), dict(l_batch=-1),
    dict(l_beam=2**41)], ids=str)
def test_select(lib, bad):
    p, need = make_select(**bad), c_size_t(0)
    assert lib.tig_beam_select_workspace_bytes(byref(p), byref(need)) == tig.TIG_EINVAL
    assert lib.tig_beam_select_run(byref(p), HOST, 1 << 40, None) == tig.TIG_EINVAL
    assert b"select" in lib.tig_last_error(None)


def test_workspaces(lib):
    need = c_size_t(0)
    c, p = make_cache(max_pages=1000), make_attend(ld_table=1000)
    assert lib.tig_cache_attend_workspace_bytes(byref(c), byref(p), byref(need)) == tig.TIG_OK and need.value > 0
    assert lib.tig_cache_attend_run(byref(c), byref(p), None, need.value, None) == tig.TIG_EINVAL
    assert lib.tig_cache_attend_run(byref(c), byref(p), HOST + 8, need.value, None) == tig.TIG_EINVAL
    assert lib.tig_cache_attend_run(byref(c), byref(p), HOST, need.value - 1, None) == tig.TIG_ENOSPACE
    assert lib.tig_cache_attend_workspace_bytes(byref(c), byref(p), None) == tig.TIG_EINVAL
    s = make_select()
    assert lib.tig_beam_select_workspace_bytes(byref(s), byref(need)) == tig.TIG_OK and need.value > 0
    assert lib.tig_beam_select_run(byref(s), None, need.value, None) == tig.TIG_EINVAL
    assert lib.tig_beam_select_run(byref(s), HOST + 128, need.value, None) == tig.TIG_EINVAL
    assert lib.tig_beam_select_run(byref(s), HOST, need.value - 1, None) == tig.TIG_ENOSPACE
    # nothing to do: no workspace, no launch
    for q in (make_attend(seqs=0, ld_table=1000, table=None, lengths=None, q=None, out=None, lse=None),):
        assert lib.tig_cache_attend_workspace_bytes(byref(c), byref(q), byref(need)) == tig.TIG_OK and need.value == 0
        assert lib.tig_cache_attend_run(byref(c), byref(q), None, 0, None) == tig.TIG_OK
    assert lib.tig_beam_select_run(byref(make_select(batch=0, logits=None)), None, 0, None) == tig.TIG_OK
    assert lib.tig_cache_append_run(byref(c), byref(make_append(seqs=0, tokens=0, ld_table=1000)), None) == tig.TIG_OK
    assert lib.tig_cache_fork_run(byref(c), byref(make_fork(rows_out=0, ld_table=1000, ld_out=1000)), None) == tig.TIG_OK


K, V = HOST, HOST + MB  # 64 * 16 * 4 * 32 * 2 bytes each
END = 64 * 16 * 4 * 32 * 2


@pytest.mark.parametrize("bad", [dict(k=K), dict(v=V + END - 2), dict(q=K - 4 * 512 - 510), dict(table=K), dict(lengths=V + 64), dict(freq=K + 8), dict(q_out=K),
                                 dict(q_out=HOST + 10 * MB), dict(q_out=HOST + 11 * MB + 64), dict(q_out=HOST + 12 * MB + 2), dict(q_out=HOST + 12 * MB, qo_token=512),
                                 dict(q_out=HOST + 8 * MB), dict(starts=V), dict(positions=K, position_type=1), dict(q_out=HOST + 14 * MB)], ids=str)
def test_append_refuses_outputs_on_top_of_others(lib, bad):
    assert lib.tig_cache_append_run(byref(make_cache()), byref(make_append(**bad)), None) == tig.TIG_EINVAL
    assert b"overlap" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", [dict(v=K), dict(v=K + END - 2), dict(k=V, v=V - END + 2), dict(v=K + 64)], ids=str)
def test_append_and_fork_refuse_values_on_top_of_keys(lib, bad):
    for call in (lambda c: lib.tig_cache_append_run(byref(c), byref(make_append()), None), lambda c: lib.tig_cache_fork_run(byref(c), byref(make_fork()), None)):
        assert call(make_cache(**bad)) == tig.TIG_EINVAL and b"overlap" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", [dict(out=K), dict(out=V + END - 2), dict(out=HOST + 10 * MB + 2), dict(out=HOST + 10 * MB, o_seq=512), dict(out=HOST + 8 * MB), dict(lse=K),
                                 dict(lse=HOST + 10 * MB), dict(lse=HOST + 11 * MB + 4), dict(lse=HOST + 9 * MB + 16)], ids=str)
def test_attend_refuses_outputs_on_top_of_others(lib, bad):
    p, need = make_attend(**bad), c_size_t(0)
    assert lib.tig_cache_attend_workspace_bytes(byref(make_cache()), byref(p), byref(need)) == tig.TIG_OK
    assert lib.tig_cache_attend_run(byref(make_cache()), byref(p), HOST, need.value, None) == tig.TIG_EINVAL
    assert b"overlap" in lib.tig_last_error(None)


@pytest.mark.parametrize("bad", [dict(table_out=HOST + 8 * MB), dict(table_out=HOST + 8 * MB + 4, ld_out=11, ld_table=11), dict(lengths_out=HOST + 9 * MB + 16),
                                 dict(table_out=K), dict(lengths_out=V), dict(table_out=HOST + 10 * MB), dict(lengths_out=HOST + 11 * MB), dict(lengths_out=HOST + 12 * MB),
                                 dict(table=V), dict(spare=K)], ids=str)
def test_fork_refuses_outputs_on_top_of_others(lib, bad):
    assert lib.tig_cache_fork_run(byref(make_cache()), byref(make_fork(**bad)), None) == tig.TIG_EINVAL
    assert b"overlap" in lib.tig_last_error(None)


OUT = ("scores_out", "parents", "tokens", "finished_out")


@pytest.mark.parametrize("out", OUT)
@pytest.mark.parametrize("on", ("logits", "scores", "finished", *OUT))
def test_select_refuses_outputs_on_top_of_others(lib, out, on):
    if out == on:
        return
    p, need = make_select(), c_size_t(0)
    setattr(p, out, getattr(p, on))
    assert lib.tig_beam_select_workspace_bytes(byref(p), byref(need)) == tig.TIG_OK
    assert lib.tig_beam_select_run(byref(p), HOST, need.value, None) == tig.TIG_EINVAL
    assert b"overlap" in lib.tig_last_error(None)


# --------------------------------------------------------------------------- the calls on tensors

CACHES = torch.zeros(8, 4, 2, 16), torch.zeros(8, 4, 2, 16)
TABLE, LENGTHS = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
ROWS, QUERIES = torch.zeros(3, 2, 16), torch.zeros(3, 4, 16)
FREQ = torch.zeros(8, dtype=torch.float64)
I32 = torch.zeros(3, dtype=torch.int32)
LOGITS, SCORES = torch.zeros(2, 3, 40), torch.zeros(2, 3)


def append(**kw):
    a = dict(k_cache=CACHES[0], v_cache=CACHES[1], table=TABLE, lengths=LENGTHS, k=ROWS, v=ROWS, q=QUERIES, freq=FREQ)
    a.update(kw)
    return ops.cache_append(**a)


def attend(**kw):
    a = dict(q=QUERIES, k_cache=CACHES[0], v_cache=CACHES[1], table=TABLE, lengths=LENGTHS)
    a.update(kw)
    return ops.cache_attend(**a)


def fork(**kw):
    a = dict(k_cache=CACHES[0], v_cache=CACHES[1], table=TABLE, lengths=LENGTHS, parents=I32, spare=I32)
    a.update(kw)
    return ops.cache_fork(**a)


def select(**kw):
    a = dict(logits=LOGITS, k=3, scores=SCORES)
    a.update(kw)
    return ops.beam_select(**a)


SHARED = {
    "3-dimensional cache": dict(k_cache=torch.zeros(8, 4, 32)), "float64 cache": dict(k_cache=CACHES[0].double(), v_cache=CACHES[1].double()),
    "values of another shape": dict(v_cache=torch.zeros(8, 4, 2, 8)), "values of another type": dict(v_cache=CACHES[1].half()),
    "values of other strides": dict(v_cache=torch.zeros(8, 2, 4, 16).transpose(1, 2)), "columns apart": dict(k_cache=torch.zeros(8, 4, 2, 32)[..., ::2], v_cache=torch.zeros(8, 4, 2, 32)[..., ::2]),
    "int64 table": dict(table=TABLE.long()), "1-dimensional table": dict(table=TABLE[0]), "table's columns apart": dict(table=torch.zeros(3, 10, dtype=torch.int32)[:, ::2]),
    "int64 lengths": dict(lengths=LENGTHS.long()), "lengths of others": dict(lengths=LENGTHS[:2]), "lengths apart": dict(lengths=torch.zeros(6, dtype=torch.int32)[::2]),
}
CALLS = [(f, kw, n) for f in (append, attend, fork) for n, kw in SHARED.items()] + [
    (append, dict(k=ROWS[0]), "2-dimensional k"), (append, dict(k=ROWS[:2], v=ROWS[:2]), "tokens without starts"), (append, dict(k=ROWS.half()), "k of another type"),
    (append, dict(v=ROWS[:, :1]), "v of other heads"), (append, dict(k=torch.zeros(3, 2, 32)[..., ::2]), "k's columns apart"), (append, dict(q=QUERIES[0]), "2-dimensional q"),
    (append, dict(q=QUERIES[..., :8]), "q of another width"), (append, dict(q=None, q_out=QUERIES), "q_out without q"), (append, dict(q_out=ROWS), "q_out of other heads"),
    (append, dict(freq=FREQ.float()), "float32 freq"), (append, dict(positions=torch.zeros(3)), "float32 positions"), (append, dict(positions=torch.zeros(2, dtype=torch.int64)), "positions of others"),
    (append, dict(starts=I32), "starts without an end"), (append, dict(starts=torch.zeros(4)), "float32 starts"),
    (attend, dict(q=QUERIES[0]), "2-dimensional q"), (attend, dict(q=QUERIES.half()), "q of another type"), (attend, dict(q=QUERIES[:2]), "q of others"),
    (attend, dict(out=ROWS), "out of other heads"), (attend, dict(out=torch.zeros(3, 4, 32)[..., ::2]), "out's columns apart"),
    (fork, dict(parents=I32.long()), "int64 parents"), (fork, dict(spare=I32[:2]), "spare of others"), (fork, dict(parents=torch.zeros(6, dtype=torch.int32)[::2]), "parents apart"),
    (select, dict(logits=LOGITS[0]), "2-dimensional logits"), (select, dict(logits=LOGITS.double()), "float64 logits"), (select, dict(logits=torch.zeros(2, 3, 80)[..., ::2]), "candidates apart"),
    (select, dict(k=0), "k 0"), (select, dict(end=40), "end behind the vocabulary"), (select, dict(end=2**40), "end far behind it"), (select, dict(end=-2), "end -2"), (select, dict(k=129), "k 129"), (select, dict(scores=SCORES[0]), "scores of others"), (select, dict(scores=SCORES.double()), "float64 scores"),
    (select, dict(finished=SCORES), "float32 finished"), (select, dict(finished=torch.zeros(2, 2, dtype=torch.bool)), "finished of others"),
    (select, dict(scores=torch.zeros(3, 2).t()), "scores in another order"),
]


@pytest.mark.parametrize("f, kw", [c[:2] for c in CALLS], ids=[f"{c[0].__name__}: {c[2]}" for c in CALLS])
def test_tensors_that_do_not_fit(f, kw):
    with pytest.raises(tig.TigError) as e:
        f(**kw)
    assert e.value.status == tig.TIG_EINVAL and "not on a GPU" not in str(e.value)


@pytest.mark.parametrize("f, names", [(append, ("k_cache", "v_cache", "k", "v", "q", "q_out", "freq")), (attend, ("q", "k_cache", "v_cache", "out")), (fork, ("k_cache", "v_cache")),
                                      (select, ("logits", "scores"))], ids=lambda x: getattr(x, "__name__", ""))
def test_tensors_that_want_a_graph_are_refused(f, names):
    given = dict(k_cache=CACHES[0], v_cache=CACHES[1], k=ROWS, v=ROWS, q=QUERIES, q_out=QUERIES, out=QUERIES, freq=FREQ, logits=LOGITS, scores=SCORES)
    for n in names:
        with pytest.raises(tig.TigError, match="no_grad") as e:
            f(**{n: given[n].clone().requires_grad_()})
        assert e.value.status == tig.TIG_EINVAL
        with torch.no_grad(), pytest.raises(tig.TigError, match="not on a GPU"):  # (the next thing that is refused here)
            f(**{n: given[n].clone().requires_grad_()})


def rows_meet(n, a, m, b, d):
    """Whether two of the rows of d columns at i a + j b, i < n, j < m, share one: row by row."""
    starts = sorted(i * a + j * b for i in range(n) for j in range(m))
    return any(y - x < d for x, y in zip(starts, starts[1:]))


@pytest.mark.parametrize("token, head", [(32, 32), (64, 32), (32, 64), (64, 64), (96, 32), (224, 32), (255, 32), (240, 48), (33, 100), (100, 50), (250, 1000), (1000, 250)], ids=str)
def test_rows_of_an_output_that_meet_are_refused(lib, token, head):
    """... where each stride alone leaves room for a row: 5 tokens (sequences) of 8 heads of 32 columns."""
    assert rows_meet(5, token, 8, head, 32)
    assert lib.tig_cache_append_run(byref(make_cache()), byref(make_append(qo_token=token, qo_head=head)), None) == tig.TIG_EINVAL
    assert b"rows of q_out overlap" in lib.tig_last_error(None)
    assert lib.tig_cache_attend_run(byref(make_cache()), byref(make_attend(o_seq=token, o_head=head)), HOST, 1 << 40, None) == tig.TIG_EINVAL
    assert b"rows of out overlap" in lib.tig_last_error(None)


def test_rows_of_an_output_that_pass_each_other_are_taken(lib):
    """Rows of one head between those of another are no overlap: what is refused next, a workspace that is missing, says so."""
    c, taken = make_cache(max_pages=1000, heads=2, head_stride=64), 0
    for seqs, q_heads in ((5, 8), (2, 2), (3, 4), (7, 2)):
        for o_seq in range(32, 330, 7):
            for o_head in range(32, 330, 9):
                p = make_attend(seqs=seqs, q_heads=q_heads, o_seq=o_seq, o_head=o_head, ld_table=1000)
                assert lib.tig_cache_attend_run(byref(c), byref(p), None, 1 << 40, None) == tig.TIG_EINVAL
                said = lib.tig_last_error(None)
                assert (b"rows of out overlap" if rows_meet(seqs, o_seq, q_heads, o_head, 32) else b"workspace is NULL") in said, (seqs, q_heads, o_seq, o_head)
                taken += b"workspace" in said
    assert taken > 100
