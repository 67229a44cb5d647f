"""Histories in a paged key-value cache, and the selection of what comes next, as cases that can be timed and compared.

Kinds of pass (the `kind` of a case):

  append  new keys and values of many sequences into their pages, keys (and the queries that come with them) rotated by their
          position on the way (ops.cache_append)
  attend  attention of one query per sequence and head over its sequence's pages (ops.cache_attend)
  select  the k best continuations over beams and vocabulary: log-probabilities on top of the beams' scores (ops.beam_select)
  fork    the selected beams take their parents' sequences over: full pages are shared, the last one is copied (ops.cache_fork)

`run` computes them with elementary torch operations, or, where `own` is true, with the framework's calls.
"""
import math

import torch

if torch.cuda.is_available():
    torch.backends.cuda.matmul.allow_tf32 = False

own = False

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


def listed():
    return [
        # one sequence that is extended by one token: latency counts
        dict(name="append_token", kind="append", seqs=1, old=999, new=1, lens="equal", qh=32, kvh=8, dim=128, page=16, dtype="bf16", rotary=128,
             interleaved=False, pos="place", head_major=False),
        # a batch of 4000 events, one for each node's history, embedding of 100 columns as two heads, positions are event times
        dict(name="append_events_fp32", kind="append", seqs=4000, old=200, new=1, lens="log", qh=2, kvh=2, dim=50, page=20, dtype="fp32", rotary=50,
             interleaved=True, pos="time", head_major=False),
        # whole prompts of different lengths behind nothing or behind a shared beginning; part of the head is rotated
        dict(name="append_prompts_fp16", kind="append", seqs=24, old=500, new=5000, lens="uniform", qh=24, kvh=8, dim=128, page=64, dtype="fp16",
             rotary=96, interleaved=False, pos="int64", head_major=True),
        # one sequence of a thousand tokens: latency counts
        dict(name="attend_token", kind="attend", seqs=1, longest=1000, lens="equal", empty=0.0, qh=32, kvh=8, dim=128, page=16, dtype="bf16", window=0,
             head_major=False),
        # every source of a batch over its node's whole history: most are short, some have thousands of events
        dict(name="attend_events_fp32", kind="attend", seqs=4000, longest=3000, lens="log", empty=0.05, qh=2, kvh=2, dim=50, page=20, dtype="fp32",
             window=0, head_major=False),
        # a service's batch in all states of progress, a key-value head for every query head
        dict(name="attend_batch_fp16", kind="attend", seqs=77, longest=4096, lens="uniform", empty=0.0, qh=16, kvh=16, dim=64, page=64, dtype="fp16",
             window=0, head_major=True),
        # few very long sequences
        dict(name="attend_long_bf16", kind="attend", seqs=4, longest=131071, lens="equal", empty=0.0, qh=64, kvh=8, dim=128, page=16, dtype="bf16",
             window=0, head_major=False),
        # four beams over a small vocabulary
        dict(name="select_token", kind="select", batch=1, beams=4, vocab=32000, k=4, dtype="bf16", finished=0.0, masked=0.0),
        # eight beams each over the nodes of the partition workload, some of them at their end, some nodes masked
        dict(name="select_nodes_bf16", kind="select", batch=50, beams=8, vocab=250_000, k=8, dtype="bf16", finished=0.1, masked=0.01),
        # the hundred best of a million candidates for every request
        dict(name="select_best_fp32", kind="select", batch=129, beams=1, vocab=1_000_003, k=100, dtype="fp32", finished=0.0, masked=0.0),
        # a few beams of a few requests
        dict(name="fork_beams", kind="fork", batch=4, beams=4, longest=1000, lens="uniform", kvh=8, dim=128, page=16, dtype="bf16", head_major=False),
        # many requests with large pages
        dict(name="fork_many_fp16", kind="fork", batch=256, beams=8, longest=500, lens="uniform", kvh=4, dim=128, page=64, dtype="fp16",
             head_major=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _shape(rng):
    """Key-value heads, query heads and their width."""
    dim = rng.choice([64, 128, 128, _log_int(rng, 8, 256)])
    kvh = rng.choice([1, 2, 4, 8, _log_int(rng, 1, 16)])
    qh = kvh * rng.choice([1, 1, 2, 4, 8, _log_int(rng, 1, 16)])
    return dict(kvh=kvh, qh=qh, dim=dim, page=rng.choice([16, 32, 64, _log_int(rng, 1, 256)]), dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]),
                head_major=rng.random() < 0.4)


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "select", "fork"])
    if kind == "select":
        vocab, batch = _log_int(rng, 100, 1_000_000), _log_int(rng, 1, 200)
        beams = rng.choice([1, 4, 8, _log_int(rng, 1, 16)])
        beams = max(1, min(beams, 100_000_000 // vocab))
        batch = max(1, min(batch, 100_000_000 // (vocab * beams)))
        return dict(kind=kind, batch=batch, beams=beams, vocab=vocab, k=rng.choice([beams, beams, _log_int(rng, 1, 100)]),
                    dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), finished=rng.choice([0.0, round(rng.uniform(0.0, 0.5), 2)]),
                    masked=rng.choice([0.0, round(rng.uniform(0.0, 0.3), 2)]))
    c = dict(_shape(rng), kind=kind, lens=rng.choice(["equal", "uniform", "log"]))
    row = c["kvh"] * c["dim"]
    if kind == "append":
        new = rng.choice([1, 1, _log_int(rng, 2, 8000)])
        c["seqs"] = max(1, min(_log_int(rng, 1, 4000), 100_000_000 // ((row + c["qh"] * c["dim"]) * (new + 300))))
        c.update(old=_log_int(rng, 1, 300), new=new)
        c["rotary"] = rng.choice([c["dim"] // 2 * 2, c["dim"] // 4 * 2, 0])
        c.update(interleaved=rng.random() < 0.3, pos=rng.choice(["place", "int64", "time"]))
        return c
    if kind == "attend":
        longest = _log_int(rng, 1, 130_000)
        longest = min(longest, 250_000_000 // row)
        c["seqs"] = max(1, min(_log_int(rng, 1, 4000), 250_000_000 // (row * longest), 32_000_000 // (c["qh"] * longest)))
        c.update(longest=longest, empty=rng.choice([0.0, 0.1]), window=rng.choice([0, 0, 0, _log_int(rng, 1, longest)]))
        return c
    c["longest"] = _log_int(rng, 1, 2000)
    c["beams"] = rng.choice([4, 8, _log_int(rng, 1, 16)])
    page_bytes = c["page"] * row
    c["batch"] = max(1, min(_log_int(rng, 1, 256), 100_000_000 // (row * (c["longest"] + c["page"])), 16_000_000 // (page_bytes * c["beams"])))
    del c["qh"]
    return c


# --------------------------------------------------------------------------- inputs


def _lengths(n, longest, how):
    """n lengths up to `longest` in ascending order (the seed only puts them into another order)."""
    if how == "equal":
        return [longest] * n
    if how == "uniform":
        return [max(1, math.ceil((i + 1) / n * longest)) for i in range(n)]
    return [max(1, min(longest, round(longest ** ((i + 1) / n)))) for i in range(n)]  # evenly over the logarithm


def _shuffled(values, gen):
    t = torch.tensor(values, dtype=torch.int64, device=DEVICE)
    return t[torch.randperm(len(values), device=DEVICE, generator=gen)]


def _cache(c, pages, normal):
    """Keys' and values' pages as [pages, page, heads, dim], the way the case wants them in memory."""
    shape = (pages, c["kvh"], c["page"], c["dim"]) if c["head_major"] else (pages, c["page"], c["kvh"], c["dim"])
    both = normal(*shape), normal(*shape)
    return [x.transpose(1, 2) if c["head_major"] else x for x in both]


def _table(lengths, width, page, gen):
    """A page of its own for every piece of every sequence, in random order; -1 behind a sequence's end."""
    need = (lengths + page - 1) // page
    pages = int(need.sum())
    order = torch.randperm(max(1, pages), device=DEVICE, generator=gen)
    inside = torch.arange(width, device=DEVICE) < need.unsqueeze(1)
    table = torch.full((lengths.numel(), width), -1, dtype=torch.int32, device=DEVICE)
    table[inside] = order[:pages].to(torch.int32)
    return table, pages


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    t = TYPES[c["dtype"]]

    def normal(*shape, std=1.0, dtype=t):
        out = torch.empty(*shape, device=DEVICE, dtype=dtype)
        flat = out.view(-1)
        for a in range(0, flat.numel(), 1 << 27):  # (large caches without a copy in 32 bits)
            n = min(1 << 27, flat.numel() - a)
            flat[a : a + n] = torch.randn(n, device=DEVICE, generator=gen) * std
        return out

    if c["kind"] == "append":
        n = c["seqs"]
        new, old = _lengths(n, c["new"], c["lens"]), _lengths(n, c["old"], c["lens"])
        most = n + (sum(new) + sum(old)) // c["page"]  # pages, however the two meet
        new = _shuffled(new, gen)
        lengths = _shuffled(old, gen) - 1 + new  # (some start empty)
        width = -(-(c["old"] + c["new"]) // c["page"])
        table, _ = _table(lengths, width, c["page"], gen)
        tokens = int(new.sum())
        k_cache, v_cache = _cache(c, most, normal)
        s = dict(case=c, k_cache=k_cache, v_cache=v_cache, table=table, lengths=lengths.to(torch.int32), starts=None, positions=None, freq=None)
        if c["new"] > 1:
            s["starts"] = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0)]).to(torch.int32)
        # as they come out of one product: queries, keys and values side by side
        qkv = normal(tokens, c["qh"] + 2 * c["kvh"], c["dim"])
        s["q"], s["k"], s["v"] = qkv[:, : c["qh"]], qkv[:, c["qh"] : c["qh"] + c["kvh"]], qkv[:, c["qh"] + c["kvh"] :]
        if c["rotary"]:
            i = torch.arange(c["rotary"] // 2, device=DEVICE, dtype=torch.float64)
            s["freq"] = 10000.0 ** (-2.0 * i / c["rotary"])
        if c["pos"] == "int64":  # counted from a beginning that is not in the cache
            s["positions"] = torch.randint(0, 1 << 20, (tokens,), device=DEVICE, generator=gen)
        elif c["pos"] == "time":  # seconds of thirty days
            s["positions"] = (torch.rand(tokens, device=DEVICE, generator=gen, dtype=torch.float64) * 30 * 86400).sort().values
        return s
    if c["kind"] == "attend":
        lengths = _shuffled(_lengths(c["seqs"], c["longest"], c["lens"]), gen)
        lengths[: int(c["empty"] * c["seqs"])] = 0
        table, pages = _table(lengths, -(-c["longest"] // c["page"]), c["page"], gen)
        k_cache, v_cache = _cache(c, max(1, pages), normal)
        return dict(case=c, q=normal(c["seqs"], c["qh"], c["dim"]), k_cache=k_cache, v_cache=v_cache, table=table, lengths=lengths.to(torch.int32))
    if c["kind"] == "select":
        # some candidates are popular whatever the request
        logits = normal(c["batch"], c["beams"], c["vocab"], std=2.0)
        logits += normal(c["vocab"], std=1.5)
        if c["masked"] > 0:
            logits.masked_fill_(torch.rand(c["vocab"], device=DEVICE, generator=gen) < c["masked"], float("-inf"))
        rows = (c["batch"], c["beams"])
        s = dict(case=c, logits=logits, scores=-20.0 * torch.rand(*rows, device=DEVICE, generator=gen), finished=None, end=-1)
        if c["finished"] > 0:
            s["finished"] = torch.rand(*rows, device=DEVICE, generator=gen) < c["finished"]
            s["end"] = 2
        return s
    rows = c["batch"] * c["beams"]
    lengths = _shuffled(_lengths(c["batch"], c["longest"], c["lens"]), gen).repeat_interleave(c["beams"])
    width = c["longest"] // c["page"] + 1
    table, pages = _table(lengths, width, c["page"], gen)
    k_cache, v_cache = _cache(c, pages + rows, normal)
    parents = torch.randint(0, c["beams"], (c["batch"], c["beams"]), device=DEVICE, generator=gen)
    parents += torch.arange(c["batch"], device=DEVICE).unsqueeze(1) * c["beams"]
    spare = pages + torch.randperm(rows, device=DEVICE, generator=gen)
    return dict(case=c, k_cache=k_cache, v_cache=v_cache, table=table, lengths=lengths.to(torch.int32), parents=parents.to(torch.int32),
                spare=spare.to(torch.int32))


# --------------------------------------------------------------------------- one pass


def _rotate(x, angle, rotary, interleaved):
    """x [tokens, heads, dim] in 32 bits, angle [tokens, rotary / 2] in 64."""
    c, s = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    r = x[..., :rotary]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    else:
        a, b = r[..., : rotary // 2], r[..., rotary // 2 :]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    return torch.cat([turned, x[..., rotary:]], dim=-1)


def _append(s):
    c = s["case"]
    t, P = TYPES[c["dtype"]], c["page"]
    lengths, n = s["lengths"].long(), c["seqs"]
    tokens = s["k"].shape[0]
    if s["starts"] is None:
        seq = torch.arange(n, device=DEVICE)
        place = lengths - 1
    else:
        starts = s["starts"].long()
        token = torch.arange(tokens, device=DEVICE)
        seq = torch.bucketize(token, starts[1:], right=True)
        place = lengths[seq] - (starts[seq + 1] - token)
    page = s["table"].long()[seq, place // P]
    k, q = s["k"].float(), s["q"].float()
    if c["rotary"]:
        pos = place.double() if s["positions"] is None else s["positions"].double()
        angle = pos.unsqueeze(1) * s["freq"]
        k, q = (_rotate(x, angle, c["rotary"], c["interleaved"]) for x in (k, q))
    s["k_cache"][page, place % P] = k.to(t)
    s["v_cache"][page, place % P] = s["v"]
    return {"k": s["k_cache"], "v": s["v_cache"], "q": q.to(t)}


def _attend(s):
    c = s["case"]
    t, P, d, kvh = TYPES[c["dtype"]], c["page"], c["dim"], c["kvh"]
    n, width = s["table"].shape
    G = c["qh"] // kvh
    lengths = s["lengths"].long()
    page = s["table"].long().clamp(min=0)
    place = torch.arange(width * P, device=DEVICE)
    k = s["k_cache"][page].reshape(n, width * P, kvh, d).float()
    score = torch.matmul(s["q"].float().view(n, kvh, G, d), k.permute(0, 2, 3, 1).contiguous()) * d**-0.5
    del k
    first = (lengths - c["window"]).clamp(min=0) if c["window"] else torch.zeros_like(lengths)
    inside = (place < lengths.unsqueeze(1)) & (place >= first.unsqueeze(1))
    score.masked_fill_(~inside.view(n, 1, 1, -1), float("-inf"))
    top = score.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    v = s["v_cache"][page].reshape(n, width * P, kvh, d).float()
    out = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()) / total.clamp(min=torch.finfo(torch.float32).tiny)
    lse = top + torch.log(total)
    return {"out": out.view(n, c["qh"], d).to(t), "lse": lse.view(n, c["qh"])}


def _select(s):
    c = s["case"]
    B, J, V, k = c["batch"], c["beams"], c["vocab"], c["k"]
    minus = float("-inf")
    x = s["logits"].double()  # (candidates of two beams may lie next to each other)
    top = x.amax(-1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(-1, keepdim=True))
    x = (x - lse) + s["scores"].double().unsqueeze(-1)
    if s["finished"] is not None:
        x.masked_fill_(s["finished"].unsqueeze(-1), minus)
        at_end = torch.where(s["finished"], s["scores"].double(), x[..., s["end"]])
        x[..., s["end"]] = at_end
    x = x.view(B, J * V)
    k_got = min(k, J * V)
    border = x.topk(k_got, dim=1).values[:, -1:]
    # all candidates down to the border in their order, so that the lowest of equal ones come first
    b, i = torch.nonzero((x >= border) & (x > minus), as_tuple=True)
    count = torch.bincount(b, minlength=B)
    most = int(count.max())
    at = torch.arange(b.numel(), device=DEVICE) - (count.cumsum(0) - count)[b]
    value = torch.full((B, max(k, most)), minus, dtype=torch.float64, device=DEVICE)
    index = torch.full((B, max(k, most)), -1, dtype=torch.int64, device=DEVICE)
    value[b, at], index[b, at] = x[b, i], i
    value, order = value.sort(dim=1, descending=True, stable=True)
    value, index = value[:, :k], index.gather(1, order)[:, :k]
    left = index >= 0
    row = torch.arange(B, device=DEVICE).unsqueeze(1) * J
    parents = torch.where(left, index // V + row, -1)
    tokens = torch.where(left, index % V, -1)
    out = {"scores": value.float(), "parents": parents.to(torch.int32), "tokens": tokens.to(torch.int32)}
    if s["finished"] is not None:
        out["finished"] = left & ((tokens == s["end"]) | s["finished"].view(-1)[parents.clamp(min=0)])
    return out


def _fork(s):
    c = s["case"]
    P = c["page"]
    parents = s["parents"].view(-1).long()
    lengths = s["lengths"].long()[parents]
    table = s["table"].long()[parents]
    full, tail = lengths // P, lengths % P
    column = torch.arange(table.shape[1], device=DEVICE)
    last = table.gather(1, full.unsqueeze(1)).squeeze(1)
    spare = s["spare"].long()
    off = torch.arange(P, device=DEVICE)
    row, at = torch.nonzero(off < tail.unsqueeze(1), as_tuple=True)
    for x in (s["k_cache"], s["v_cache"]):
        x[spare[row], at] = x[last[row], at]
    table = torch.where(column < full.unsqueeze(1), table, torch.where(column == full.unsqueeze(1), spare.unsqueeze(1), -1))
    return {"k": s["k_cache"], "v": s["v_cache"], "table": table.to(torch.int32), "lengths": lengths.to(torch.int32)}


def _own(s):
    from paper_2308_14129_amd import ops

    c = s["case"]
    if c["kind"] == "append":
        q = ops.cache_append(s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["k"], s["v"], starts=s["starts"], q=s["q"], freq=s["freq"],
                             positions=s["positions"], interleaved=c["interleaved"])
        return {"k": s["k_cache"], "v": s["v_cache"], "q": q}
    if c["kind"] == "attend":
        out, lse = ops.cache_attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], window=c["window"], lse=True)
        return {"out": out, "lse": lse}
    if c["kind"] == "select":
        r = ops.beam_select(s["logits"], c["k"], s["scores"], finished=s["finished"], end=s["end"])
        out = {"scores": r.scores, "parents": r.parents, "tokens": r.tokens}
        if s["finished"] is not None:
            out["finished"] = r.finished
        return out
    table, lengths = ops.cache_fork(s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["parents"], s["spare"])
    return {"k": s["k_cache"], "v": s["v_cache"], "table": table, "lengths": lengths}


def run(state):
    if own:
        return _own(state)
    return {"append": _append, "attend": _attend, "select": _select, "fork": _fork}[state["case"]["kind"]](state)


# --------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    """Inputs read once, outputs written once: new keys, values and queries and their places; the keys and values that a query sees;
    the logits; the pages that are copied.  A rotated pair takes 6 operations, a key that a query sees 4 a column, a logit
    about 4."""
    c = dict(case)
    size = SIZE[c["dtype"]]
    if c["kind"] == "append":
        tokens = sum(_lengths(c["seqs"], c["new"], c["lens"]))
        return {"bytes": 2.0 * tokens * (c["qh"] + 2 * c["kvh"]) * c["dim"] * size + 8.0 * c["seqs"],
                "flops": 3.0 * tokens * (c["qh"] + c["kvh"]) * c["rotary"] + 1.0}
    if c["kind"] == "attend":
        lens = _lengths(c["seqs"], c["longest"], c["lens"])
        keys = sum(min(l, c["window"]) if c["window"] else l for l in lens) * (1.0 - int(c["empty"] * c["seqs"]) / c["seqs"])
        return {"bytes": 2.0 * keys * c["kvh"] * c["dim"] * size + c["seqs"] * c["qh"] * (2.0 * c["dim"] * size + 4) + 4.0 * keys / c["page"],
                "flops": 4.0 * keys * c["qh"] * c["dim"]}
    if c["kind"] == "select":
        rows = c["batch"] * c["beams"]
        return {"bytes": 1.0 * rows * (c["vocab"] * size + 4) + 12.0 * c["batch"] * c["k"], "flops": 4.0 * rows * c["vocab"]}
    rows = c["batch"] * c["beams"]
    tails = sum(l % c["page"] for l in _lengths(c["batch"], c["longest"], c["lens"])) * c["beams"]
    return {"bytes": 4.0 * tails * c["kvh"] * c["dim"] * size + 8.0 * rows * (c["longest"] // c["page"] + 3), "flops": 1.0 * rows}


# --------------------------------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    f64 = torch.float64
    if c["kind"] == "append":
        P, r = c["page"], c["rotary"]
        k_cache, v_cache = s["k_cache"].to(f64), s["v_cache"].to(f64)
        x = torch.cat([s["k"], s["q"]], dim=1).to(f64)
        lengths = s["lengths"].tolist()
        starts = list(range(c["seqs"] + 1)) if s["starts"] is None else s["starts"].tolist()
        table = s["table"].cpu()
        slots, places = [], []
        for i, total in enumerate(lengths):
            p = torch.arange(total - (starts[i + 1] - starts[i]), total)
            places.append(p)
            slots.append(table[i, p // P].long() * P + p % P)
        places, slots = torch.cat(places).to(DEVICE), torch.cat(slots).to(DEVICE)
        if r:
            pos = places.to(f64) if s["positions"] is None else s["positions"].to(f64)
            turn = torch.polar(torch.ones((), dtype=f64, device=DEVICE), torch.outer(pos, s["freq"]))[:, None, :]
            first = x[..., 0:r:2] if c["interleaved"] else x[..., : r // 2]
            second = x[..., 1:r:2] if c["interleaved"] else x[..., r // 2 : r]
            z = torch.complex(first.contiguous(), second.contiguous()) * turn
            first.copy_(z.real)  # (views of x)
            second.copy_(z.imag)
        k_cache[slots // P, slots % P] = x[:, : c["kvh"]]
        v_cache[slots // P, slots % P] = s["v"].to(f64)
        return {"k": k_cache, "v": v_cache, "q": x[:, c["kvh"] :].contiguous()}
    if c["kind"] == "attend":
        P, d, G = c["page"], c["dim"], c["qh"] // c["kvh"]
        out = torch.zeros(c["seqs"], c["qh"], d, dtype=f64, device=DEVICE)
        lse = torch.full((c["seqs"], c["qh"]), float("-inf"), dtype=f64, device=DEVICE)
        for i, total in enumerate(s["lengths"].tolist()):
            first = max(0, total - c["window"]) if c["window"] else 0
            if total <= first:
                continue
            pages = s["table"][i, first // P : -(-total // P)].long()
            cut = slice(first % P, first % P + total - first)
            for h in range(c["kvh"]):
                k = s["k_cache"][pages, :, h].reshape(-1, d)[cut].to(f64)
                v = s["v_cache"][pages, :, h].reshape(-1, d)[cut].to(f64)
                a = torch.mm(s["q"][i, h * G : (h + 1) * G].to(f64), k.t().contiguous()) / math.sqrt(d)
                out[i, h * G : (h + 1) * G] = torch.mm(torch.softmax(a, -1), v)
                lse[i, h * G : (h + 1) * G] = torch.logsumexp(a, -1)
        return {"out": out, "lse": lse}
    if c["kind"] == "select":
        B, J, V, k = c["batch"], c["beams"], c["vocab"], c["k"]
        scores = torch.full((B, k), float("-inf"), dtype=f64, device=DEVICE)
        parents = torch.full((B, k), -1, dtype=torch.int32, device=DEVICE)
        tokens, done = parents.clone(), torch.zeros(B, k, dtype=torch.bool, device=DEVICE)
        fin = torch.zeros(B, J, dtype=torch.bool, device=DEVICE) if s["finished"] is None else s["finished"]
        for b in range(B):
            found = []
            logp = torch.log_softmax(s["logits"][b].to(f64), -1)
            for j in range(J):
                base = float(s["scores"][b, j].to(f64))
                if bool(fin[b, j]):
                    found.append((-base, j, s["end"], True))
                    continue
                best = torch.topk(logp[j], min(k, V)).values
                at = torch.nonzero(logp[j] >= best[-1]).flatten()
                for v, l in zip(at.tolist(), logp[j][at].tolist()):
                    if l > float("-inf"):
                        found.append((-(base + l), j, v, v == s["end"]))
            found.sort()
            for n, (value, j, v, last) in enumerate(found[:k]):
                scores[b, n], parents[b, n], tokens[b, n], done[b, n] = -value, b * J + j, v, last
        out = {"scores": scores, "parents": parents, "tokens": tokens}
        if s["finished"] is not None:
            out["finished"] = done
        return out
    P = c["page"]
    k_cache, v_cache = s["k_cache"].to(f64), s["v_cache"].to(f64)
    old, lengths, parents, spare = s["table"].tolist(), s["lengths"].tolist(), s["parents"].flatten().tolist(), s["spare"].tolist()
    table, new = [], []
    for row, p in enumerate(parents):
        total = lengths[p]
        new.append(total)
        n, left = total // P, total % P
        table.append(old[p][:n] + [spare[row]] + [-1] * (len(old[p]) - n - 1))
        if left:
            k_cache[spare[row], :left] = k_cache[old[p][n], :left]
            v_cache[spare[row], :left] = v_cache[old[p][n], :left]
    return {"k": k_cache, "v": v_cache, "table": torch.tensor(table, dtype=torch.int32, device=DEVICE),
            "lengths": torch.tensor(new, dtype=torch.int32, device=DEVICE)}
