"""Paged caches for the tests: pages in random order, whatever no sequence has filled with NaN, several orders in memory."""
import torch

DEV = "cuda:0"
F64 = torch.float64
U = 2.0**-24
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
LAYOUTS = ("rows", "heads", "outer", "kv", "pairs", "padded")


def half(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    return torch.finfo(t).tiny * torch.finfo(t).eps / 2


def gen_of(seed, device=DEV):
    return torch.Generator(device=device).manual_seed(seed)


def make_cache(pages, size, heads, dim, t, layout, fill=float("nan"), device=DEV):
    """Keys' and values' pages as [pages, size, heads, dim] views of `layout`."""
    def full(*shape):
        return torch.full(shape, fill, dtype=t, device=device)

    if layout == "rows":
        return full(pages, size, heads, dim), full(pages, size, heads, dim)
    if layout == "heads":
        return full(pages, heads, size, dim).transpose(1, 2), full(pages, heads, size, dim).transpose(1, 2)
    if layout == "outer":
        return full(heads, pages, size, dim).permute(1, 2, 0, 3), full(heads, pages, size, dim).permute(1, 2, 0, 3)
    if layout == "kv":
        return full(pages, 2, size, heads, dim).unbind(1)
    if layout == "pairs":
        return full(pages, size, heads, 2, dim).unbind(3)
    both = full(2, pages * (size * heads * (dim + 3) + 5) + 1)  # one element into the allocation, gaps everywhere
    return tuple(x[1:].as_strided((pages, size, heads, dim), (size * heads * (dim + 3) + 5, heads * (dim + 3), dim + 3, 1), x.storage_offset() + 1)
                 for x in both.unbind(0))


def make_table(lengths, size, width, spare, gen):
    """A table of random distinct pages, junk behind each sequence's; `spare` pages more than are used."""
    device = gen.device
    need = [-(-n // size) for n in lengths]
    pages = max(1, sum(need) + spare)
    order = torch.randperm(pages, generator=gen, device=device).tolist()
    table = torch.randint(-5, pages + 5, (len(lengths), width), generator=gen, device=device, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        if n:
            table[i, :n] = torch.tensor(order[at : at + n], dtype=torch.int32)
        at += n
    return table, pages, order[at:]


def gather(cache, table, i, lo, hi):
    """Rows lo .. hi - 1 of sequence i as [rows, heads, dim] in fp64; rows on no page are None in the mask."""
    pages, size = cache.shape[:2]
    p = torch.arange(lo, hi, device=cache.device)
    page = table[i].long()[p // size]
    ok = (page >= 0) & (page < pages)
    return cache[page.clamp(0, pages - 1), p % size].to(F64), ok


def close(got, ref, tol, name):
    got = got.to(F64)
    bad = ~((got - ref).abs() <= tol) & ~(torch.isnan(got) & torch.isnan(ref)) & ~(got == ref)
    if bad.any():
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])} for {float(ref[i])}, tolerance {float((tol + 0 * ref)[i])}")


def attention(q, k_cache, v_cache, table, lengths, scale, window):
    """out, lse in fp64 and bounds of their errors, by the formula.

    A score is a sum of d fp32 products (d + 2 operations), scaled; a weight is an fp32 exponential (4 units) of a difference whose
    rounding is two units of its size; two 16-bit parts hold a weight to 2^-17; sums over a sequence's rows and their joins add a
    unit for every row."""
    n, qh, d = q.shape
    pages, size, kvh, _ = k_cache.shape
    cap = table.shape[1] * size
    t = q.dtype
    out = torch.zeros(n, qh, d, dtype=F64, device=q.device)
    lse = torch.full((n, qh), float("-inf"), dtype=F64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    for i in range(n):
        end = min(max(int(lengths[i]), 0), cap)
        first = max(0, end - window) if window else 0
        if end == first:
            continue
        k, ok = gather(k_cache, table, i, first, end)
        v, _ = gather(v_cache, table, i, first, end)
        if not ok.any():
            continue
        k, v = k[ok], v[ok]
        G = qh // kvh
        Q = q[i].to(F64).view(kvh, G, d)
        K, V = k.permute(1, 0, 2).contiguous(), v.permute(1, 0, 2).contiguous()
        s = scale * torch.matmul(Q, K.transpose(1, 2).contiguous())
        size_s = abs(scale) * torch.matmul(Q.abs(), K.abs().transpose(1, 2).contiguous())
        l = torch.logsumexp(s, -1, keepdim=True)
        p = torch.exp(s - l)
        off = (2 * (d + 3) * U * size_s).amax(-1, keepdim=True) + 4 * U * (s - s.amax(-1, keepdim=True)).abs() + (k.shape[0] + 32) * U
        if t is not torch.float32:
            off = off + 2.0**-17
        o = torch.matmul(p, V)
        lost = torch.matmul(p * off, V.abs()) + o.abs() * (p * off).sum(-1, keepdim=True)
        out[i], lse[i] = o.reshape(qh, d), l.reshape(qh)
        tol[i] = (half(t) * o.abs() + 1.01 * lost + tiny(t)).reshape(qh, d)
        tol_lse[i] = 1.01 * ((p * off).sum(-1).reshape(qh) + 8 * U * (l.abs() + s.abs().amax(-1, keepdim=True)).reshape(qh))
    return out, lse, tol, tol_lse
