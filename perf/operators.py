"""The operators of a trained head as a user's program calls them, as cases that can be timed and compared.

Kinds of pass (the `kind` of a case):

  linear  a dense layer with bias, activation and residual in one call (ops.linear); with `train` its backward pass too
          (ops.linear_backward): gradients of the input, the matrix and the bias
  loss    softmax cross entropy over a vocabulary of candidates (ops.softmax_ce): loss and log-sum-exp of every row, with
          `grad` the gradients of rows, candidates' matrix and candidates' bias
  adamw   one optimiser step over many tensors (ops.AdamW): states in 32 bits, or in 8 as values of four exponent and three
          mantissa bits with a power of two for every 256

`run` computes them with elementary torch operations, or, where `own` is true, with the framework's calls.
"""
import math

import numpy as np
import torch

if torch.cuda.is_available():
    torch.backends.cuda.matmul.allow_tf32 = False

own = False

DEVICE = "cuda:0"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BLOCK = 256  # values of an 8-bit state that share a scale

# Row widths of the model: [state | time] 172 + 100, embedding 100 (tensors of the medium datasets' configuration).
MEDIUM = dict(mem=172, time=100, feat=172, emb=100)


def listed():
    return [
        # one embedding at a time through a layer of a scoring service: the matrix is read once, latency counts
        dict(name="linear_token", kind="linear", rows=1, inp=1024, out=4096, dtype="bf16", act="gelu", residual=False, train=False),
        # a few requests at a time, odd widths
        dict(name="linear_serve_13", kind="linear", rows=13, inp=2000, out=1333, dtype="fp16", act="silu", residual=True, train=False),
        # merge layer of the partition workload: [attention | state] 300 -> 100 for the 12000 queries of a batch
        dict(name="linear_merge_fp32", kind="linear", rows=12000, inp=300, out=100, dtype="fp32", act="relu", residual=False, train=True),
        # a block's feed-forward layer in a training batch
        dict(name="linear_train_bf16", kind="linear", rows=8192, inp=4096, out=16384, dtype="bf16", act="gelu", residual=True, train=True),
        # a batch of 200 over the thousand items of the medium dataset, widths of its embedding
        dict(name="loss_medium_fp32", kind="loss", rows=200, vocab=1000, dim=100, dtype="fp32", bias=True, scale=1.0, ignored=0.1, grad=True),
        # a batch of the partition workload over all the nodes that are seen there
        dict(name="loss_nodes_bf16", kind="loss", rows=4000, vocab=250_000, dim=100, dtype="bf16", bias=True, scale=1.0, ignored=0.05, grad=True),
        # ranking loss of a validation batch over a million candidates, no gradient
        dict(name="loss_score_fp16", kind="loss", rows=999, vocab=1_000_003, dim=128, dtype="fp16", bias=False, scale=1.0, ignored=0.0, grad=False),
        # a large vocabulary under wide rows
        dict(name="loss_wide_bf16", kind="loss", rows=8192, vocab=128_000, dim=2048, dtype="bf16", bias=False, scale=1.0, ignored=0.02, grad=True),
        # the model's own 22 tensors, with clipping
        dict(MEDIUM, name="adamw_model", kind="adamw", blocks=0, width=0, table=0, dtype="fp32", master=False, bits=32, max_norm=1.0),
        # a table of candidates and a few blocks, 16-bit tensors beside 32-bit masters
        dict(name="adamw_blocks_bf16", kind="adamw", mem=0, time=0, feat=0, emb=0, blocks=12, width=1024, table=32_000, dtype="bf16", master=True,
             bits=32, max_norm=1.0),
        # the same kind with 8-bit states, without clipping
        dict(name="adamw_blocks_8bit", kind="adamw", mem=0, time=0, feat=0, emb=0, blocks=10, width=1000, table=100_000, dtype="bf16", master=True,
             bits=8, max_norm=0.0),
        # a candidates' table of the partition workload: one long fp32 tensor with 8-bit states
        dict(name="adamw_table_8bit", kind="adamw", mem=0, time=0, feat=0, emb=0, blocks=1, width=100, table=250_000, dtype="fp32", master=False,
             bits=8, max_norm=1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "loss", "adamw"])
    if kind == "linear":
        train = rng.random() < 0.6
        rows, inp, out = _log_int(rng, 1, 16384), _log_int(rng, 16, 4096), _log_int(rng, 16, 16384)
        if rng.random() < 0.4:
            inp, out = -(-inp // 64) * 64, -(-out // 64) * 64
        act = rng.choice(["none", "relu", "gelu", "silu"])
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        rows = max(1, min(rows, 500_000_000_000 // (inp * out) if dtype != "fp32" else 100_000_000_000 // (inp * out)))
        return dict(kind=kind, rows=rows, inp=inp, out=out, dtype=dtype, act=act, residual=rng.random() < 0.5, train=train)
    if kind == "loss":
        grad = rng.random() < 0.75
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        vocab, dim = _log_int(rng, 500, 1_000_000), _log_int(rng, 32, 2048)
        if rng.random() < 0.4:
            vocab, dim = -(-vocab // 128) * 128, -(-dim // 64) * 64
        most = 1_500_000_000_000 if dtype != "fp32" else 200_000_000_000
        rows = max(1, min(_log_int(rng, 1, 8192), 1_000_000_000 // vocab, most // (vocab * dim)))
        return dict(kind=kind, rows=rows, vocab=vocab, dim=dim, dtype=dtype, bias=rng.random() < 0.5,
                    scale=1024.0 if dtype == "fp16" else 1.0, ignored=round(rng.choice([0.0, rng.uniform(0.0, 0.5)]), 3), grad=grad)
    model = rng.random() < 0.4
    dtype = "fp32" if model else rng.choice(["bf16", "fp16", "fp32"])
    blocks = 0 if model else rng.randint(1, 8)
    c = dict(kind=kind, mem=_log_int(rng, 32, 172) if model else 0, time=_log_int(rng, 16, 100) if model else 0,
             feat=_log_int(rng, 4, 172) if model else 0, emb=_log_int(rng, 32, 128) if model else 0, blocks=blocks,
             width=0 if model else _log_int(rng, 50, 1024), table=0 if model else _log_int(rng, 1000, 60_000), dtype=dtype,
             master=dtype != "fp32", bits=rng.choice([8, 32]), max_norm=rng.choice([0.0, 1.0]))
    return c


# --------------------------------------------------------------------------- inputs


def _sizes(c):
    """Element counts of an optimiser's tensors, and whether each is a vector (which takes no weight decay)."""
    if c["mem"]:
        M, T, F, E = c["mem"], c["time"], c["feat"], c["emb"]
        da, dkv, D = M + T, M + F + T, 2 * M + T + F
        n = [T, T, 3 * M * D, 3 * M, 3 * M * M, 3 * M, da * da, da, da * dkv, da, da * dkv, da, da * da, da, E * (da + M), E, E * E, E, E * 2 * E, E, E, 1]
        vec = [True, True] + [False, True] * 9 + [True, True]
        return n, vec
    w = c["width"]
    n, vec = [c["table"] * w], [False]
    for _ in range(c["blocks"]):
        n += [w * w] * 4 + [4 * w * w] * 2 + [w] * 6 + [4 * w]
        vec += [False] * 6 + [True] * 7
    return n, vec


LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    t = TYPES[c["dtype"]]

    def normal(*shape, std=1.0, dtype=t):
        return (torch.randn(*shape, device=DEVICE, generator=gen) * std).to(dtype)

    if c["kind"] == "linear":
        s = dict(case=c, x=normal(c["rows"], c["inp"]), w=normal(c["out"], c["inp"], std=c["inp"] ** -0.5), bias=normal(c["out"], std=0.1),
                 residual=normal(c["rows"], c["out"]) if c["residual"] else None)
        if c["train"]:
            s["dy"] = normal(c["rows"], c["out"])
        return s
    if c["kind"] == "loss":
        n, V = c["rows"], c["vocab"]
        s = dict(case=c, x=normal(n, c["dim"]), w=normal(V, c["dim"], std=1.5 * c["dim"] ** -0.5), bias=normal(V, std=0.3) if c["bias"] else None)
        # few candidates draw most of the answers, as a hub does
        u = torch.rand(n, device=DEVICE, generator=gen, dtype=torch.float64)
        labels = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
        if c["ignored"] > 0:
            labels[torch.rand(n, device=DEVICE, generator=gen) < c["ignored"]] = -1
        s["labels"] = labels.to(torch.int32)
        return s
    n, vec = _sizes(c)
    starts, at = [], 0
    for k in n:
        starts.append(at)
        at += -(-k // BLOCK) * BLOCK
    inside = torch.zeros(at + 1, device=DEVICE, dtype=torch.int32)
    inside[torch.tensor(starts, device=DEVICE)] += 1
    inside.index_add_(0, torch.tensor([a + k for a, k in zip(starts, n)], device=DEVICE),
                      torch.full((len(n),), -1, device=DEVICE, dtype=torch.int32))
    inside = inside.cumsum(0)[:at] > 0

    def flat(std, dtype=torch.float32, square=False):
        x = torch.randn(at, device=DEVICE, generator=gen) * std * inside
        return (x * x if square else x).to(dtype)

    s = dict(case=c, n=n, starts=starts, vec=vec, master=flat(0.02), grad=flat(0.01, t), m=flat(0.003), v=flat(0.01, square=True),
             step=torch.full((1,), 99, dtype=torch.int64, device=DEVICE))
    s["param"] = s["master"].to(t) if c["master"] else s["master"]
    decay = torch.zeros(at, device=DEVICE)
    for a, k, flag in zip(starts, n, vec):
        if not flag:
            decay[a : a + k] = DECAY
    s["decay"] = decay
    if c["bits"] == 8:
        nb = at // BLOCK
        for name, x in (("m", s["m"]), ("v", s["v"].sqrt())):
            x = x.view(nb, BLOCK)
            top = x.abs().amax(1, keepdim=True)
            scale = torch.where(top > 0, torch.exp2(torch.floor(torch.log2(top.double())) - 7.0).float(), torch.ones_like(top))
            s[name] = (x / scale).to(torch.float8_e4m3fn).view(-1)
            s[name + "_scale"] = scale.view(-1)
    return s


# --------------------------------------------------------------------------- one pass


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return g * (1.0 + z * (1.0 - g))
    return torch.ones_like(z)


def _linear(s):
    c = s["case"]
    t, act = TYPES[c["dtype"]], c["act"]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t() + s["bias"].float()
    y = _act(z, act)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if not c["train"]:
        return {"y": y.to(t)}
    dz = s["dy"].float() * _act_slope(z, act)
    return {"y": y.to(t), "dx": (dz @ w).to(t), "dw": (dz.t() @ x).to(t), "db": dz.sum(0).to(t)}


def _loss(s):
    c = s["case"]
    t = TYPES[c["dtype"]]
    x, w, labels = s["x"].float(), s["w"].float(), s["labels"].long()
    logits = x @ w.t()
    if s["bias"] is not None:
        logits += s["bias"].float()
    counted = labels >= 0
    at = labels.clamp(min=0).unsqueeze(1)
    top = logits.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(logits - top).sum(1, keepdim=True))
    loss = torch.where(counted, (lse - logits.gather(1, at)).squeeze(1), torch.zeros_like(top.squeeze(1)))
    count = counted.sum()
    out = {"loss": loss, "lse": lse.squeeze(1), "mean": (loss.double().sum() / count.clamp(min=1)).float().view(1)}
    if c["grad"]:
        scale = torch.where(counted, c["scale"] / count.clamp(min=1).float(), torch.zeros_like(loss)).unsqueeze(1)
        p = torch.exp(logits - lse)
        p.scatter_add_(1, at, torch.full_like(lse, -1.0))
        p *= scale
        out.update(dx=(p @ w).to(t), dw=(p.t() @ x).to(t))
        if s["bias"] is not None:
            out["dbias"] = p.sum(0).to(t)
    return out


def _to_8bit(x, u, positive):
    """Blocks of values as e4m3 values and a power of two each: up or down by the threshold u of the place in the block."""
    top = x.abs().amax(1, keepdim=True)
    scale = torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.frexp(top)[1] - 8), torch.ones_like(top))
    y = x.abs() / scale
    e = torch.frexp(y)[1].clamp(min=-5) - 4
    q = torch.ldexp(torch.floor(torch.ldexp(y, -e) + u), e)
    q = torch.where(x > 0, q.clamp(min=2.0**-9), q) if positive else torch.where(x < 0, -q, q)
    return q.to(torch.float8_e4m3fn).view(-1), scale.view(-1)


def _adamw(s):
    c = s["case"]
    s["step"] += 1
    t = s["step"].double()
    g = s["grad"].float()
    if c["max_norm"] > 0:
        norm = s["grad"].double().square().sum().sqrt()
        g = g * (c["max_norm"] / norm).clamp(max=1.0).float()
    eight = c["bits"] == 8
    nb = g.numel() // BLOCK
    if eight:
        m = (s["m"].float().view(nb, BLOCK) * s["m_scale"].view(nb, 1)).view(-1)
        r = (s["v"].float().view(nb, BLOCK) * s["v_scale"].view(nb, 1)).view(-1)
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + (g * g) * (1.0 - BETA2)
    root = v.sqrt()
    step_size = (LR / (1.0 - BETA1**t)).float()
    root_scale = (1.0 / (1.0 - BETA2**t).sqrt()).float()
    p = s["master"] * (1.0 - LR * s["decay"]) - step_size * (m / (root * root_scale + EPS))
    s["master"].copy_(p)
    if c["master"]:
        s["param"].copy_(p)
    if not eight:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return _adamw_out(s)
    place = torch.arange(BLOCK, device=DEVICE) * 0x6A09E667 + s["step"] * 0x9E3779B9
    u = ((place & 0xFFFFFFFF) >> 8).float() * 2.0**-24
    half = (((place + 0x80000000) & 0xFFFFFFFF) >> 8).float() * 2.0**-24
    for name, x, at, positive in (("m", m, u, False), ("v", root, half, True)):
        q, scale = _to_8bit(x.view(nb, BLOCK), at, positive)
        s[name].copy_(q)
        s[name + "_scale"].copy_(scale)
    return _adamw_out(s)


def _adamw_out(s):
    out = {"master": s["master"], "m": s["m"], "v": s["v"]}
    if s["case"]["master"]:
        out["param"] = s["param"]
    if s["case"]["bits"] == 8:
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    return out


def _own(s):
    from paper_2308_14129_amd import ops

    c = s["case"]
    if c["kind"] == "linear":
        y = ops.linear(s["x"], s["w"], s["bias"], s["residual"], c["act"], keep=c["train"])
        if not c["train"]:
            return {"y": y}
        y, z = y
        dx, dw, db = ops.linear_backward(s["dy"], s["x"], s["w"], z, c["act"])
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if c["kind"] == "loss":
        r = ops.softmax_ce(s["x"], s["w"], s["labels"], s["bias"], scale=c["scale"], grad=c["grad"])
        out = {"loss": r.loss, "lse": r.lse, "mean": r.mean}
        if c["grad"]:
            out.update(dx=r.dx, dw=r.dw)
            if s["bias"] is not None:
                out["dbias"] = r.dbias
        return out
    if "opt" not in s:  # the handle that a training program makes once
        def parts(x, size=1):
            return [x[a // size : a // size + -(-k // size)] for a, k in zip(s["starts"], s["n"])]

        eight = c["bits"] == 8
        s["opt"] = ops.AdamW(parts(s["param"]), parts(s["grad"]), parts(s["m"]), parts(s["v"]), s["step"],
                             masters=parts(s["master"]) if c["master"] else None,
                             m_scales=parts(s["m_scale"], BLOCK) if eight else None, v_scales=parts(s["v_scale"], BLOCK) if eight else None,
                             betas=(BETA1, BETA2), eps=EPS, weight_decay=[0.0 if flag else DECAY for flag in s["vec"]])
    s["opt"].step(LR, max_norm=c["max_norm"])
    return _adamw_out(s)


def run(state):
    if own:
        return _own(state)
    return {"linear": _linear, "loss": _loss, "adamw": _adamw}[state["case"]["kind"]](state)


# --------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    """Inputs read once, outputs written once.  A layer's product is 2 rows inp out flops, twice that again for its gradients;
    the loss' logits, and its two gradients, 2 rows vocab dim each; an optimiser's step about 16 operations an element."""
    c = dict(case)
    size = 4 if c["dtype"] == "fp32" else 2
    if c["kind"] == "linear":
        r, i, o = c["rows"], c["inp"], c["out"]
        b = size * (r * i + i * o + o + r * o * (2 if c["residual"] else 1))
        f = 2.0 * r * i * o
        if c["train"]:
            b += size * (r * o + r * i + i * o + o)
            f *= 3
        return {"bytes": b, "flops": f}
    if c["kind"] == "loss":
        n, V, d = c["rows"], c["vocab"], c["dim"]
        vec = V if c["bias"] else 0
        b = size * (n * d + V * d + vec) + 4 * n * 3
        f = 2.0 * n * V * d
        if c["grad"]:
            b += size * (n * d + V * d + vec)
            f *= 3
        return {"bytes": b, "flops": f}
    n = sum(_sizes(c)[0])
    each = 8 + size + (size if c["master"] else 0) + (4 + 16 / BLOCK if c["bits"] == 8 else 16)
    return {"bytes": n * each, "flops": 16.0 * n}


# --------------------------------------------------------------------------- the definition in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    f64 = torch.float64
    if c["kind"] == "linear":
        x, w = s["x"].to(f64), s["w"].to(f64)
        z = torch.addmm(s["bias"].to(f64), x, w.t())
        phi = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        sig = torch.sigmoid(z)
        value = {"none": z, "relu": torch.relu(z), "gelu": z * phi, "silu": z * sig}[c["act"]]
        y = value if s["residual"] is None else value + s["residual"].to(f64)
        if not c["train"]:
            return {"y": y}
        density = torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
        slope = {"none": torch.ones_like(z), "relu": torch.heaviside(z, torch.zeros((), dtype=f64, device=z.device)),
                 "gelu": phi + z * density, "silu": sig + z * sig * (1 - sig)}[c["act"]]
        dz = s["dy"].to(f64) * slope
        return {"y": y, "dx": torch.mm(dz, w), "dw": torch.mm(dz.t(), x), "db": dz.sum(0)}
    if c["kind"] == "loss":
        x, w, labels = s["x"].to(f64), s["w"].to(f64), s["labels"].long()
        logits = torch.mm(x, w.t()) if s["bias"] is None else torch.addmm(s["bias"].to(f64), x, w.t())
        lse = torch.logsumexp(logits, 1)
        rows = torch.nonzero(labels >= 0).flatten()
        loss = torch.zeros_like(lse)
        loss[rows] = lse[rows] - logits[rows, labels[rows]]
        out = {"loss": loss, "lse": lse, "mean": loss.sum().view(1) / max(1, rows.numel())}
        if c["grad"]:
            g = torch.exp(logits[rows] - lse[rows, None])
            del logits
            g[torch.arange(rows.numel(), device=g.device), labels[rows]] -= 1.0
            g *= c["scale"] / max(1, rows.numel())
            dx = torch.zeros_like(x)
            dx[rows] = torch.mm(g, w)
            out.update(dx=dx, dw=torch.mm(g.t(), x[rows]))
            if s["bias"] is not None:
                out["dbias"] = g.sum(0)
        return out
    t = int(s["step"]) + 1
    g = s["grad"].to(f64)
    if c["max_norm"] > 0:
        g = g * min(1.0, c["max_norm"] / float(torch.linalg.vector_norm(g)))
    if c["bits"] == 8:
        m = (s["m"].to(f64).view(-1, BLOCK) * s["m_scale"].to(f64)[:, None]).flatten()
        v = (s["v"].to(f64).view(-1, BLOCK) * s["v_scale"].to(f64)[:, None]).flatten().square()
    else:
        m, v = s["m"].to(f64), s["v"].to(f64)
    m = torch.lerp(g, m, BETA1)
    v = torch.lerp(g.square(), v, BETA2)
    m_hat, v_hat = m / (1 - BETA1**t), v / (1 - BETA2**t)
    p = s["master"].to(f64)
    p = p - LR * (s["decay"].to(f64) * p + m_hat / (v_hat.sqrt() + EPS))
    # what is held in 8 bits goes up or down by a threshold: it has no value in 64 bits of its own
    out = {"master": p, "m": m if c["bits"] == 32 else None, "v": v if c["bits"] == 32 else None}
    if c["master"]:
        out["param"] = p
    if c["bits"] == 8:
        out.update(m_scale=None, v_scale=None)
    return out
