"""Operators around the prompt in a paged cache of full precision: what is measured, and their plain forms.

Kinds of pass (`case["kind"]`):

  chunk     keys and values of new tokens stored into their pages, then attention of these tokens over all of their sequence
  sums      attention weights of new tokens added up for every cached position
  evict     the cache of a batch cut to a budget by those sums, all layers
  logprobs  log probability, rank and entropy for given tokens, with the most probable alternatives

The cache: pools [page][KV head][row of the page][d] and a block table; a slot is page * page size + row in the page.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ---------------------------------------------------------------------------- cases
def _chunk(name, B, H_q, H_kv, d, dtype, lo, hi, n_lo, n_hi, prompts, page):
    """B sequences with prefixes spread over [lo, hi]; every prompts-th one brings n_lo..n_hi new tokens, the others one."""
    return {"name": name, "kind": "chunk", "B": B, "H_q": H_q, "H_kv": H_kv, "d": d, "dtype": dtype, "lo": lo, "hi": hi,
            "n_lo": n_lo, "n_hi": n_hi, "prompts": prompts, "page": page}


def _sums(name, B, H_q, H_kv, d, dtype, lo, hi, n_lo, n_hi, prompts, page, last):
    return {**_chunk(name, B, H_q, H_kv, d, dtype, lo, hi, n_lo, n_hi, prompts, page), "kind": "sums", "last": last}


def _evict(name, B, layers, H_kv, d, dtype, lo, hi, keep, first, recent, page, fresh):
    return {"name": name, "kind": "evict", "B": B, "layers": layers, "H_kv": H_kv, "d": d, "dtype": dtype, "lo": lo, "hi": hi,
            "keep": keep, "first": first, "recent": recent, "page": page, "fresh": fresh}


def _logprobs(name, rows, V, dtype, top, mapped, masked):
    return {"name": name, "kind": "logprobs", "rows": rows, "V": V, "dtype": dtype, "top": top, "mapped": mapped, "masked": masked}


def listed():
    return [
        # a draft model that decodes token after token: one short sequence, small heads; launches and latency
        _chunk("chunk_token_d64", 1, 12, 12, 64, "bf16", 517, 517, 1, 1, 1, 64),
        # plain decoding of a batch of chats, grouped heads: all bytes, few rows per KV head
        _chunk("chunk_decode_gqa", 32, 32, 8, 128, "bf16", 100, 8000, 1, 1, 1, 64),
        # continuous batching: most sequences decode, every eighth brings a piece of its prompt
        _chunk("chunk_mixed", 32, 32, 8, 128, "bf16", 64, 4096, 200, 512, 8, 64),
        # prompts of a batch from their first token on, one head of queries per head of keys
        _chunk("chunk_prompts", 8, 32, 32, 128, "bf16", 0, 0, 1000, 2048, 1, 64),
        # a piece of a long document behind what is cached of it, grouped heads (heads and length of workload c5)
        _chunk("chunk_long_gqa", 1, 64, 8, 128, "bf16", 16384, 16384, 2048, 2048, 1, 128),
        # the weights of a decoded token per sequence join the sums (every layer of a decode round does this)
        _sums("sums_decode", 32, 32, 8, 128, "bf16", 100, 8000, 1, 1, 1, 64, 0),
        # a prompt's last rows decide what of it is kept
        _sums("sums_prompt_tail", 4, 32, 8, 128, "bf16", 2000, 7000, 1024, 1024, 1, 64, 64),
        # one sequence, one layer, in place: a little over its budget
        _evict("evict_single", 1, 1, 8, 128, "bf16", 1200, 1200, 1024, 4, 128, 64, False),
        # a batch, several layers, the pages of the long form stay with another owner
        _evict("evict_batch", 16, 8, 8, 128, "bf16", 2048, 8192, 1024, 4, 256, 64, True),
        # the tokens that one step of one sequence has emitted
        _logprobs("logprobs_step", 6, 32000, "fp32", 5, True, False),
        # rows under a grammar, half precision head, odd vocabulary
        _logprobs("logprobs_masked", 240, 50001, "bf16", 20, False, True),
        # all tokens of prompts that are scored
        _logprobs("logprobs_prompt", 4096, 32000, "fp32", 20, False, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _bounded(make, *most):
    """A case made by `make` whose work is at most the most of the cases `most`."""
    limits = [work(c) for c in most]
    while True:
        case = make()
        w = work(case)
        if all(w[k] <= max(limit[k] for limit in limits) for k in ("bytes", "flops")):
            return {k: v for k, v in case.items() if k != "name"}


def draw(rng):
    kind = rng.choice(("chunk", "chunk", "chunk", "sums", "evict", "logprobs"))
    by_name = {c["name"]: c for c in listed()}

    def batch():
        H_kv = rng.choice((1, 2, 4, 5, 8, 12, 32))
        d = rng.choice((32, 64, 80, 96, 128, 128, 128, 256))
        hi = rng.choice((0, _log(rng, 1, 16384), _log(rng, 1, 16384)))
        n = _log(rng, 1, 2048)
        return (_log(rng, 1, 32), H_kv * rng.choice((1, 1, 2, 4, 7, 8)), H_kv, d, rng.choice(("bf16", "bf16", "bf16", "fp32")),
                rng.choice((hi, hi // 16, 0)), hi, max(1, n // rng.choice((1, 2, 8))), n, rng.choice((1, 1, 3, 8)), rng.choice((32, 64, 96, 128, 256)))

    def evict():
        hi = _log(rng, 1, 16384)
        return _evict("", _log(rng, 1, 32), _log(rng, 1, 16), rng.choice((1, 2, 5, 8, 32)), rng.choice((32, 64, 80, 96, 128, 256)),
                      rng.choice(("bf16", "fp32")), rng.choice((hi, max(1, hi // 8))), hi, _log(rng, 1, 4096), rng.choice((0, 1, 4)),
                      rng.choice((0, 16, 256)), rng.choice((32, 64, 96, 128)), rng.random() < 0.5)

    if kind == "chunk":
        return _bounded(lambda: _chunk("", *batch()), by_name["chunk_long_gqa"], by_name["chunk_decode_gqa"])
    if kind == "sums":
        return _bounded(lambda: _sums("", *batch(), rng.choice((0, 1, 64))), by_name["sums_prompt_tail"], by_name["sums_decode"])
    if kind == "evict":
        return _bounded(evict, by_name["evict_batch"])
    return _bounded(lambda: _logprobs("", _log(rng, 1, 4096), rng.choice((_log(rng, 64, 262144), 32000, 50001, 151936)),
                                      rng.choice(("bf16", "fp32")), rng.choice((0, 1, 5, 20, 32)), rng.random() < 0.3, rng.random() < 0.3),
                    by_name["logprobs_prompt"])


def _spread(b):
    return (b * 0.6180339887498949) % 1.0


def lengths(case):
    """Cached tokens of a batch, spread over [lo, hi], the longest first, in a fixed order."""
    return [case["hi"] - int(math.floor((case["hi"] - case["lo"]) * _spread(b))) for b in range(case["B"])]


def chunks(case):
    """New tokens of every sequence of a batch."""
    n = [case["n_hi"] - int(math.floor((case["n_hi"] - case["n_lo"]) * _spread(b + 3))) for b in range(case["B"])]
    return [n[b] if b % case["prompts"] == 0 else 1 for b in range(case["B"])]


def _size(case):
    return 4 if case["dtype"] == "fp32" else 2


def work(case):
    kind = case["kind"]
    if kind in ("chunk", "sums"):
        H_q, H_kv, d, size = case["H_q"], case["H_kv"], case["d"], _size(case)
        cached = new = used = pairs = 0
        for L, n in zip(lengths(case), chunks(case)):
            w = n if kind == "chunk" or not case["last"] else min(n, case["last"])
            cached, new, used = cached + L, new + n, used + w
            pairs += w * (L + n) - w * (w - 1) // 2
        if kind == "chunk":
            # new keys and values are read as rows, written to their pages and not needed from there again
            return {"bytes": size * (2 * H_kv * d * (cached + 2 * new) + 2 * H_q * d * new), "flops": 4 * d * H_q * pairs}
        return {"bytes": size * d * (H_kv * (cached + new) + H_q * used) + 4 * H_q * used + 4 * H_kv * (2 * cached + new), "flops": 2 * d * H_q * pairs}
    if kind == "evict":
        read = kept = 0
        for n in lengths(case):
            m = min(n, case["keep"])
            read, kept = read + n, kept + m
        heads = case["layers"] * case["H_kv"]
        return {"bytes": heads * (4 * read + kept * (4 * case["d"] * _size(case) + 8)), "flops": 4 * heads * read}
    return {"bytes": case["rows"] * (case["V"] * _size(case) + 8 * case["top"] + 16), "flops": 6 * case["rows"] * case["V"]}


# ---------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _randn(g, dtype, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _tables(case, totals, g):
    """Pages in random order; a block table with -1 behind a sequence's last page."""
    page = case["page"]
    need = [-(-n // page) for n in totals]
    width, n_pages = max(1, max(need)), sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).int()
    table = torch.full((len(totals), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    return table, n_pages


def _slots(table, page, start, stop):
    pos = torch.arange(start, stop, device=DEV)
    return table[pos // page].int() * page + (pos % page).int()


def _prepare_chunk(case, seed):
    g = _generator(seed)
    dtype, H_q, H_kv, d, page = _dtype(case), case["H_q"], case["H_kv"], case["d"], case["page"]
    L, n = lengths(case), chunks(case)
    totals = [a + b for a, b in zip(L, n)]
    table, n_pages = _tables(case, totals, g)
    T = sum(n)
    start = [0]
    for k in n:
        start.append(start[-1] + k)
    st = {"case": case, "host_len": L, "host_start": start, "prefix_len": _ints(L), "chunk_start": _ints(start), "table": table,
          "capacity": table.shape[1] * page, "scale": 1.0 / math.sqrt(d),
          "k_pool": _randn(g, dtype, n_pages, H_kv, page, d)}
    if case["kind"] == "chunk":
        # queries, keys and values as they leave one fused projection
        fused = _randn(g, dtype, T, (H_q + 2 * H_kv) * d)
        st["q"] = fused[:, :H_q * d].view(T, H_q, d)
        st["k_new"] = fused[:, H_q * d:(H_q + H_kv) * d].view(T, H_kv, d)
        st["v_new"] = fused[:, (H_q + H_kv) * d:].view(T, H_kv, d)
        st["v_pool"] = _randn(g, dtype, n_pages, H_kv, page, d)
        st["slot_map"] = torch.cat([_slots(table[b], page, L[b], totals[b]) for b in range(case["B"])])
        st["out"] = torch.empty(T, H_q, d, dtype=dtype, device=DEV)
        st["lse"] = torch.empty(T, H_q, dtype=torch.float32, device=DEV)
        if own:
            from paper_2401_06706_amd import binding as M
            st["store"] = M.store_args(st["k_new"], st["v_new"], st["slot_map"], st["k_pool"], st["v_pool"])
            need = M.mcsd_chunk_workspace_bytes(M.chunk_desc(st["q"], st["k_pool"], table, st["scale"], st["capacity"]))
            st["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
            st["attn"] = M.chunk_attn_args(st["q"], st["k_pool"], st["v_pool"], table, st["chunk_start"], st["prefix_len"], st["out"],
                                           st["scale"], st["capacity"], st["lse"], st["ws"])
        return st
    st["q"] = _randn(g, dtype, T, H_q, d)
    # (log-sum-exp as the attention of the same rows has left it)
    st["lse"] = torch.zeros(T, H_q, dtype=torch.float32, device=DEV)
    for b in range(case["B"]):
        for h, rows, s in _scores(st, b, torch.float32, case["last"]):
            st["lse"][rows, h] = torch.logsumexp(s, -1).t()
    st["pristine"] = torch.rand(case["B"], H_kv, st["capacity"], generator=g, device=DEV) ** 4
    st["sums"] = torch.empty_like(st["pristine"])
    if own:
        from paper_2401_06706_amd import binding as M
        st["args"] = M.weight_sums_args(st["q"], st["k_pool"], table, st["chunk_start"], st["prefix_len"], st["lse"], st["sums"], st["scale"],
                                        case["last"])
    return st


def _prepare_evict(case, seed):
    g = _generator(seed)
    B, layers, H_kv, d, page, dtype = case["B"], case["layers"], case["H_kv"], case["d"], case["page"], _dtype(case)
    L = lengths(case)
    kept = [min(n, case["keep"]) for n in L]
    table, n_pages = _tables(case, L + kept, g)
    capacity = max(1, -(-max(L) // page)) * page
    table, fresh = table[:B, :capacity // page].contiguous(), table[B:, :capacity // page].contiguous()
    sums = 20.0 * torch.rand(layers, B, H_kv, capacity, generator=g, device=DEV) ** 6
    sums = torch.where(sums < 1e-3, torch.zeros_like(sums), sums)          # (positions that nothing looks at any more)
    if fresh.shape[1] < capacity // page:
        fresh = torch.cat((fresh, torch.full((B, capacity // page - fresh.shape[1]), -1, dtype=torch.int32, device=DEV)), 1)
    k, v = (_randn(g, dtype, layers, n_pages, H_kv, page, d) for _ in range(2))
    st = {"case": case, "host_len": L, "lens0": _ints(L), "prefix_len": _ints(L), "keep_len": _ints([case["keep"]] * B), "table": table,
          "fresh": fresh if case["fresh"] else None, "k_pool": k, "v_pool": v, "sums0": sums, "sums": torch.empty_like(sums),
          "kept": torch.full((layers, B, H_kv, capacity), -1, dtype=torch.int32, device=DEV),
          "flags": torch.zeros(B, dtype=torch.int32, device=DEV), "capacity": capacity}
    if not case["fresh"]:
        st["k0"], st["v0"] = k.clone(), v.clone()
    if own:
        from paper_2401_06706_amd import binding as M
        st["args"] = M.evict_args(k, v, table, st["sums"], st["prefix_len"], st["keep_len"], st["kept"], st["flags"], case["first"], case["recent"],
                                  st["fresh"])
    return st


def _prepare_logprobs(case, seed):
    g = _generator(seed)
    R, V, n = case["rows"], case["V"], min(case["top"], case["V"])
    logits = 3.0 * torch.randn(R + (5 if case["mapped"] else 0), V, generator=g, device=DEV)
    if case["masked"]:
        # a grammar leaves between some 64 tokens and all of them
        share = torch.rand(logits.shape[0], 1, generator=g, device=DEV) ** 8
        mask = torch.rand(logits.shape, generator=g, device=DEV) >= share
        mask[:, torch.randperm(V, generator=g, device=DEV)[:64]] = False
        logits = logits.masked_fill_(mask, float("-inf"))
    logits = logits.to(_dtype(case))
    temperature = 0.5 + torch.rand(R, generator=g, device=DEV)
    row_map = torch.randperm(logits.shape[0], generator=g, device=DEV)[:R].int() if case["mapped"] else None
    tokens = torch.empty(R, dtype=torch.int32, device=DEV)
    for r in range(0, R, 512):                              # tokens as they are sampled
        at = slice(r, r + 512)
        z = (logits[at][:R - r] if row_map is None else logits[row_map[at].long()]).float() / temperature[at, None]
        tokens[at] = (z - torch.log(-torch.log(torch.rand(z.shape, generator=g, device=DEV).clamp(1e-9, 1.0 - 1e-7)))).argmax(-1).int()
    st = {"case": case, "logits": logits, "tokens": tokens, "temperature": temperature, "row_map": row_map,
          "logprob": torch.empty(R, device=DEV), "entropy": torch.empty(R, device=DEV), "rank": torch.empty(R, dtype=torch.int32, device=DEV),
          "top_tok": torch.empty(R, n, dtype=torch.int32, device=DEV) if n else None, "top_logprob": torch.empty(R, n, device=DEV) if n else None,
          "flags": torch.empty(R, dtype=torch.int32, device=DEV)}
    if own:
        from paper_2401_06706_amd import binding as M
        d = M.logprob_desc(logits, st["tokens"], n)
        need = M.mcsd_logprob_workspace_bytes(d)
        st["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
        st["args"] = M.logprob_args(logits, st["tokens"], st["logprob"], st["entropy"], st["rank"], st["top_tok"], st["top_logprob"], st["flags"],
                                    st["temperature"], st["row_map"], st["ws"])
    return st


def prepare(case, seed):
    return {"chunk": _prepare_chunk, "sums": _prepare_chunk, "evict": _prepare_evict, "logprobs": _prepare_logprobs}[case["kind"]](case, seed)


# ---------------------------------------------------------------------------- one pass
def _rows_of(pool, table, page, n):
    """Rows [H_kv][n][d] of a sequence, positions 0..n-1."""
    pages = table[:-(-n // page)].long()
    return pool[pages].transpose(0, 1).reshape(pool.shape[1], -1, pool.shape[3])[:, :n]


def _scores(st, b, dtype, last=0):
    """Per KV head: (query heads, rows of q, scores [G][rows][keys] with -infinity where a row does not see a key); the keys in `dtype`."""
    case = st["case"]
    s0, s1, L = st["host_start"][b], st["host_start"][b + 1], st["host_len"][b]
    n, G = s1 - s0, case["H_q"] // case["H_kv"]
    if n == 0:
        return
    lo = max(0, n - last) if last else 0
    k = _rows_of(st["k_pool"], st["table"][b], case["page"], L + n).to(dtype)
    unseen = torch.arange(L + n, device=DEV)[None, :] > L + torch.arange(lo, n, device=DEV)[:, None]
    rows = slice(s0 + lo, s1)
    for g in range(case["H_kv"]):
        heads = slice(g * G, (g + 1) * G)
        q = st["q"][rows, heads].to(dtype).transpose(0, 1).reshape(-1, case["d"])
        s = (q @ k[g].t()).view(G, n - lo, L + n) * st["scale"]
        yield heads, rows, s.masked_fill_(unseen, float("-inf"))


def _attention(st, dtype, out, lse):
    """Attention of every sequence's new rows in `dtype`, rounded once into out."""
    case = st["case"]
    G = case["H_q"] // case["H_kv"]
    for b in range(case["B"]):
        n = st["host_len"][b] + st["host_start"][b + 1] - st["host_start"][b]
        v = _rows_of(st["v_pool"], st["table"][b], case["page"], n).to(dtype)
        for heads, rows, s in _scores(st, b, dtype):
            m = s.amax(-1, keepdim=True)
            p = torch.exp(s - m)
            total = p.sum(-1, keepdim=True)
            o = (p.reshape(-1, n) @ v[heads.start // G]).view(G, -1, case["d"]) / total
            out[rows, heads] = o.transpose(0, 1).to(out.dtype)
            lse[rows, heads] = (m + torch.log(total)).squeeze(-1).t().to(lse.dtype)


def _run_chunk(st):
    case = st["case"]
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_kv_store_paged(st["store"])
        M.mcsd_chunk_attn_paged(st["attn"])
        return st["out"], st["lse"], st["k_pool"], st["v_pool"]
    slot = st["slot_map"].long()
    page, row = slot // case["page"], slot % case["page"]
    st["k_pool"][page, :, row] = st["k_new"]
    st["v_pool"][page, :, row] = st["v_new"]
    _attention(st, torch.float32, st["out"], st["lse"])
    return st["out"], st["lse"], st["k_pool"], st["v_pool"]


def _run_sums(st):
    case = st["case"]
    st["sums"].copy_(st["pristine"])
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_attn_weight_sums(st["args"])
        return st["sums"]
    G = case["H_q"] // case["H_kv"]
    for b in range(case["B"]):
        L = st["host_len"][b]
        n = L + st["host_start"][b + 1] - st["host_start"][b]
        st["sums"][b, :, L:n] = 0.0
        for heads, rows, s in _scores(st, b, torch.float32, case["last"]):
            w = torch.exp(s - st["lse"][rows, heads].t().unsqueeze(-1))
            st["sums"][b, heads.start // G, :n] += w.sum((0, 1))
    return st["sums"]


def _order(values):
    """Indices by value, the largest first, equal ones by index."""
    return torch.sort(values, dim=-1, descending=True, stable=True).indices


def _run_evict(st):
    case = st["case"]
    st["sums"].copy_(st["sums0"])
    st["prefix_len"].copy_(st["lens0"])
    if not case["fresh"]:
        st["k_pool"].copy_(st["k0"])
        st["v_pool"].copy_(st["v0"])
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_kv_evict_paged(st["args"])
    else:
        _evict_plain(st)
    return st["k_pool"], st["v_pool"], st["sums"], st["kept"], st["prefix_len"]


def _evict_plain(st):
    case = st["case"]
    page = case["page"]
    for b, n in enumerate(st["host_len"]):
        m = min(n, case["keep"])
        old = _slots(st["table"][b], page, 0, n).long()
        new = _slots(st["table"][b] if st["fresh"] is None else st["fresh"][b], page, 0, m).long()
        # what is always kept counts as larger than all others, the first tokens ahead of the last ones
        f = min(case["first"], m)
        r = min(case["recent"], m - f)
        key = st["sums"][:, b, :, :n].clone()
        key[..., :f] = float("inf")
        key[..., n - r:] = float("inf")
        kept = torch.sort(_order(key)[..., :m]).values if m < n else torch.arange(n, device=DEV).expand(key.shape)
        st["kept"][:, b, :, :m] = kept.int()
        st["sums"][:, b, :, :m] = torch.gather(st["sums"][:, b, :, :n], -1, kept)
        src = old[kept]                                     # [layers][H_kv][m]
        layer = torch.arange(case["layers"], device=DEV)[:, None, None]
        head = torch.arange(case["H_kv"], device=DEV)[None, :, None]
        for pool in (st["k_pool"], st["v_pool"]):
            rows = pool[layer, src // page, head, src % page]
            pool[layer, new // page, head, new % page] = rows
        st["prefix_len"][b] = m


def _run_logprobs(st):
    names = ("logprob", "entropy", "rank", "top_tok", "top_logprob")
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_token_logprobs(st["args"])
        return {k: st[k] for k in names if st[k] is not None}
    n = 0 if st["top_tok"] is None else st["top_tok"].shape[1]
    for lo in range(0, st["case"]["rows"], 512):
        at = slice(lo, lo + 512)
        raw = st["logits"][at] if st["row_map"] is None else st["logits"][st["row_map"][at].long()]
        raw = raw.float()
        z = raw / st["temperature"][at, None]
        z = z - z.amax(-1, keepdim=True)
        lse = torch.log(torch.exp(z).sum(-1, keepdim=True))
        p = torch.exp(z - lse)
        tok = st["tokens"][at].long()[:, None]
        st["logprob"][at] = (torch.gather(z, 1, tok) - lse)[:, 0]
        st["entropy"][at] = (lse - torch.where(p > 0, p * z, torch.zeros_like(p)).sum(-1, keepdim=True))[:, 0]
        mine = torch.gather(raw, 1, tok)
        ids = torch.arange(raw.shape[1], device=DEV)[None]
        st["rank"][at] = ((raw > mine) | ((raw == mine) & (ids < tok))).sum(-1).int()
        if n:
            best = _order(raw)[:, :n]
            st["top_tok"][at] = best.int()
            st["top_logprob"][at] = torch.gather(z, 1, best) - lse
    return {k: st[k] for k in names if st[k] is not None}


def run(state):
    return {"chunk": _run_chunk, "sums": _run_sums, "evict": _run_evict, "logprobs": _run_logprobs}[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------- from the definitions, in 64 bits
def _exact_pairs(st, b, g, last):
    """(rows of q, query heads, 64-bit scores [rows][G][keys], keys seen [rows][1][keys], slots) a block of rows at a time."""
    case = st["case"]
    s0, s1, L = st["host_start"][b], st["host_start"][b + 1], st["host_len"][b]
    G, page = case["H_q"] // case["H_kv"], case["page"]
    slots = _slots(st["table"][b], page, 0, L + s1 - s0).long()
    keys = st["k_pool"][slots // page, g, slots % page].double()
    step = max(1, (1 << 27) // (G * keys.shape[0]))
    for r0 in range(max(s0, s1 - last) if last else s0, s1, step):
        r1 = min(s1, r0 + step)
        q = st["q"][r0:r1, g * G:(g + 1) * G].double()
        s = (q.reshape(-1, case["d"]) @ keys.t()).view(r1 - r0, G, -1) * st["scale"]
        seen = torch.arange(keys.shape[0], device=DEV) <= (L - s0 + torch.arange(r0, r1, device=DEV))[:, None, None]
        yield slice(r0, r1), slice(g * G, (g + 1) * G), s, seen, slots


def exact(case, seed):
    global own
    mode, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = mode
    kind = case["kind"]
    if kind == "chunk":
        page = case["page"]
        for t, slot in enumerate(st["slot_map"].tolist()):
            st["k_pool"][slot // page, :, slot % page] = st["k_new"][t]
            st["v_pool"][slot // page, :, slot % page] = st["v_new"][t]
        out, lse = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV), torch.zeros(st["q"].shape[:2], dtype=torch.float64, device=DEV)
        for b in range(case["B"]):
            for g in range(case["H_kv"]):
                for rows, heads, s, seen, slots in _exact_pairs(st, b, g, 0):
                    total = torch.logsumexp(torch.where(seen, s, -math.inf), -1)
                    weight = torch.where(seen, torch.exp(s - total[..., None]), 0.0)
                    values = st["v_pool"][slots // page, g, slots % page].double()
                    out[rows, heads] = (weight.reshape(-1, len(slots)) @ values).view(*weight.shape[:2], -1)
                    lse[rows, heads] = total
        return out, lse, None, None
    if kind == "sums":
        sums = st["pristine"].double()
        for b in range(case["B"]):
            L = st["host_len"][b]
            sums[b, :, L:L + st["host_start"][b + 1] - st["host_start"][b]] = 0.0
            for g in range(case["H_kv"]):
                for rows, heads, s, seen, slots in _exact_pairs(st, b, g, case["last"]):
                    weight = torch.where(seen, torch.exp(s - st["lse"][rows, heads].double()[..., None]), 0.0)
                    sums[b, g, :len(slots)] += weight.sum((0, 1))
        return sums
    if kind == "evict":
        return None                                     # (nothing here is computed: values are moved)
    n = 0 if st["top_tok"] is None else st["top_tok"].shape[1]
    out = {"logprob": [], "entropy": [], "rank": None}
    if n:
        out.update(top_tok=None, top_logprob=[])
    for r in range(case["rows"]):
        row = st["logits"][r if st["row_map"] is None else int(st["row_map"][r])].double() / st["temperature"][r].double()
        lp = torch.log_softmax(row, 0)
        out["logprob"].append(lp[st["tokens"][r].long()])
        out["entropy"].append(-(torch.exp(lp) * lp.clamp(min=-1e4)).sum())
        if n:
            out["top_logprob"].append(torch.topk(lp, n).values)
    return {k: torch.stack(v) if v is not None else None for k, v in out.items()}
