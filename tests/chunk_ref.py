"""Chunk attention over a paged cache, weight sums, eviction and token log probabilities from their definitions, in 64 bits, for
the tests; and how far fp32 arithmetic may be off."""
import math

import torch

F24 = 2.0 ** -24


def make_batch(g, dev, dtype, lens, news, H_q, H_kv, d, page, pool_pages=0, spread=0.0):
    """A packed batch over a paged cache in random page order; q as a strided slice of a wider row."""
    totals = [a + b for a, b in zip(lens, news)]
    need = [-(-n // page) for n in totals]
    n_pages = max(sum(need) + 2, pool_pages)
    width = max(1, max(need))
    order = torch.randperm(n_pages, generator=g)[:sum(need)].int()
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    T = sum(news)
    rnd = lambda *s: torch.randn(*s, generator=g).to(dtype).to(dev)
    fused = rnd(T, H_q * d + 8)
    start = [0]
    for n in news:
        start.append(start[-1] + n)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    # (every row of the pool that belongs to nobody is NaN: nothing may read it into a result)
    k = torch.full((n_pages, H_kv, page, d), float("nan"), dtype=dtype, device=dev)
    v = k.clone()
    for b, n in enumerate(totals):
        for j in range(need[b]):
            r = min(page, n - j * page)
            k[table[b, j], :, :r] = rnd(H_kv, r, d) * (1 + spread)
            v[table[b, j], :, :r] = rnd(H_kv, r, d)
    return {"lens": lens, "news": news, "start": start, "q": fused[:, :H_q * d].view(T, H_q, d), "k_pool": k, "v_pool": v, "table": table.to(dev),
            "prefix_len": i32(lens), "chunk_start": i32(start), "page": page, "capacity": width * page}


def rows_of(pool, table, page, n):
    """Rows float64 [H_kv][n][d] of a sequence; pages outside the pool are zeros."""
    out = torch.zeros(pool.shape[1], n, pool.shape[3], dtype=torch.float64, device=pool.device)
    for j in range(-(-n // page)):
        p = int(table[j])
        if 0 <= p < pool.shape[0]:
            r = min(page, n - j * page)
            out[:, j * page:j * page + r] = pool[p, :, :r].double()
    return out


def scores(batch, b, scale, lo=0):
    """Per KV head: (scores [G][rows][keys] float64, seen [rows][keys], sum |q k| scale [G][rows][keys]) of new tokens lo.. of sequence b."""
    s0, L, n = batch["start"][b], batch["lens"][b], batch["news"][b]
    k = rows_of(batch["k_pool"], batch["table"][b], batch["page"], L + n)
    H_kv, keys = k.shape[0], L + n
    q = batch["q"][s0 + lo:s0 + n].double()
    G = q.shape[1] // H_kv
    i = torch.arange(lo, n, device=k.device)
    seen = torch.arange(keys, device=k.device)[None] <= L + i[:, None]
    for h in range(H_kv):
        qh = q[:, h * G:(h + 1) * G].transpose(0, 1)
        yield (qh @ k[h].t()) * scale, seen, (qh.abs() @ k[h].abs().t()) * scale


def attention(batch, scale, dtype):
    """out, lse in 64 bits and bounds for the kernel's error of both."""
    q = batch["q"]
    d = q.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    lse_bound = torch.zeros_like(lse)
    half_step = 2.0 ** -8 if dtype == torch.bfloat16 else F24
    weight = 0.0 if dtype == torch.float32 else (2.0 ** -8 if d == 128 else 2.0 ** -16)
    for b in range(len(batch["lens"])):
        s0, n, keys = batch["start"][b], batch["news"][b], batch["lens"][b] + batch["news"][b]
        if n == 0:
            continue
        v = rows_of(batch["v_pool"], batch["table"][b], batch["page"], keys)
        G = q.shape[1] // v.shape[0]
        for g, (s, seen, mag) in enumerate(scores(batch, b, scale)):
            s = s.masked_fill(~seen, -math.inf)
            L = torch.logsumexp(s, -1)
            p = torch.exp(s - L[..., None])
            # a score: d products summed in fp32, scaled, taken from the maximum, each a rounding of what is there
            ds = (mag.masked_fill(~seen, 0).amax(-1) * (d + 4) + 4 * L.abs() + 8) * F24
            # weights e^(s - lse) off by 2 ds, sums over the keys by a rounding each
            rel = 2 * ds + (keys + 16) * F24
            o, mass = p @ v[g], p @ v[g].abs()
            at = (slice(s0, s0 + n), slice(g * G, (g + 1) * G))
            out[at], lse[at] = o.transpose(0, 1), L.t()
            bound[at] = ((rel[..., None] + weight) * mass * (1 + half_step) + half_step * o.abs() + 1e-30).transpose(0, 1)
            lse_bound[at] = (rel + 4 * F24 * (1 + L.abs())).t()
    return out, bound, lse, lse_bound


def weight_sums(batch, scale, lse, sums, last):
    """sums after the call in 64 bits and a bound for the kernel's error."""
    new = sums.double().clone()
    bound = torch.zeros_like(new)
    d = batch["q"].shape[2]
    for b in range(len(batch["lens"])):
        s0, L, n = batch["start"][b], batch["lens"][b], batch["news"][b]
        if n == 0:
            continue
        new[b, :, L:L + n] = 0.0
        old = new[b, :, :L + n].abs().clone()
        lo = max(0, n - last) if last else 0
        for g, (s, seen, mag) in enumerate(scores(batch, b, scale, lo)):
            G = s.shape[0]
            l = lse[s0 + lo:s0 + n, g * G:(g + 1) * G].double().t()[..., None]
            w = torch.exp(s - l).masked_fill(~seen, 0)
            rel = (mag * (d + 4) + 4 * l.abs() + 4 * s.abs() + 8).masked_fill(~seen, 0) * F24
            new[b, g, :L + n] += w.sum((0, 1))
            bound[b, g, :L + n] = (w * rel).sum((0, 1)) * 1.01 + (G * (n - lo) + 70) * F24 * w.sum((0, 1)) + 2 * F24 * old[g] + 1e-30
    return new, bound


def evicted(n, keep, first, recent, sums):
    """Positions kept, ascending (sums: a list of floats)."""
    m = min(n, max(0, keep))
    if m == n:
        return list(range(n))
    f = min(first, m)
    r = min(recent, m - f)
    order = sorted(range(f, n - r), key=lambda j: (-sums[j] if sums[j] == sums[j] else math.inf, sums[j] != sums[j], j))
    return sorted(list(range(f)) + order[:m - f - r] + list(range(n - r, n)))


def logprobs(row, x, T, n_top):
    """(logprob, entropy, rank, top ids, top logprobs) of a row in 64 bits; None for what has no value."""
    z = row.double()
    V = z.shape[0]
    if torch.isnan(z).any() or (z == math.inf).any() or (z == -math.inf).all():
        return None
    order = sorted(range(V), key=lambda i: (-float(z[i]), i)) if V <= 4096 else torch.sort(z, descending=True, stable=True).indices.tolist()
    lp = torch.log_softmax(z / (T if T > 0 else 1.0), 0)
    p = torch.exp(lp)
    entropy = float(-(p * lp.clamp(min=-1e5)).sum())
    known = 0 <= x < V
    rank = int(((z > z[x]) | ((z == z[x]) & (torch.arange(V, device=z.device) < x))).sum()) if known else -1
    return (float(lp[x]) if known else math.nan, entropy, rank, order[:n_top], [float(lp[i]) for i in order[:n_top]])


def logprob_bound(V, value, spread):
    """fp32 sums of a 512th of the row per lane, each term with its exponent's rounding; `spread` = (max - z) / T of the token."""
    return ((3 * V / 512 + 64) + 4 * math.log2(V + 1)) * F24 + 4 * F24 * (abs(value) + spread)
