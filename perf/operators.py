"""Operators around a prefix cache held in 4 bits: what is measured, and their plain forms.

Kinds of pass (`case["kind"]`):

  attn    tree attention of one layer over a paged cache held in 4 bits (one candidate = a single token)
  rows    keys and values of prompt tokens stored into that cache by slot and read back as rows
  commit  the accepted paths of a verification step join that cache, all layers; the rows read back
  pages   block tables, slot map and free list of a batch, from the requests' lengths
  logits  penalties, biases and grammar masks on the logit rows of the candidate trees

The cache: a row of d values is d / 32 blocks of 32 codes (sign, two exponent bits, one mantissa bit:
0, 0.5, 1, 1.5, 2, 3, 4, 6) with one scale 2^(s - 127) each.  Codes lie as [page][KV head][page size / 16][d / 32][16 rows][16 bytes],
scales as [page][KV head][page size / 16][d / 32][16 rows]; value 2i of a block is the low half of byte i.
"""
import math

import torch

own = False

DEV = "cuda:0"
CODE_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
BLOCK, TILE = 32, 16


# ---------------------------------------------------------------------------- cases
def _attn(name, B, H_q, H_kv, d, lo, hi, tree, page):
    return {"name": name, "kind": "attn", "B": B, "H_q": H_q, "H_kv": H_kv, "d": d, "lo": lo, "hi": hi, "tree": tree, "page": page}


def _rows(name, T, H_kv, d, dtype, page, fused):
    return {"name": name, "kind": "rows", "T": T, "H_kv": H_kv, "d": d, "dtype": dtype, "page": page, "fused": fused}


def _commit(name, B, layers, H_kv, d, tree, page, L):
    return {"name": name, "kind": "commit", "B": B, "layers": layers, "H_kv": H_kv, "d": d, "tree": tree, "page": page, "L": L}


def _pages(name, B, page, prompt, live):
    return {"name": name, "kind": "pages", "B": B, "page": page, "prompt": prompt, "live": live}


def _logits(name, B, tree, V, dtype, hist, mask, bias):
    return {"name": name, "kind": "logits", "B": B, "tree": tree, "V": V, "dtype": dtype, "hist": hist, "mask": mask, "bias": bias}


def listed():
    return [
        # a draft model that decodes token after token: one short sequence, small heads; launch and latency
        _attn("attn_token_d64", 1, 12, 12, 64, 517, 517, "1", 64),
        # plain decoding of a batch of chats, grouped heads: all bytes, one row per query head
        _attn("attn_decode_gqa", 32, 32, 8, 128, 100, 8000, "1", 64),
        # batched serving with candidate trees (workload c4), cache in 4 bits
        _attn("attn_tree_batch", 16, 32, 32, 128, 256, 4096, "4x2x2x1x1", 64),
        # long prompts, grouped heads and 84 candidates (workload c5): 672 rows share a KV head
        _attn("attn_tree_long", 4, 64, 8, 128, 16384, 16384, "4x4x2x1", 128),
        # a short prompt in fp32, small heads, odd length
        _rows("rows_short_fp32", 33, 8, 64, "fp32", 64, False),
        # prompts of a batch, packed, keys and values as they leave a fused projection (strided rows)
        _rows("rows_prompts", 16384, 8, 128, "bf16", 64, True),
        # one interactive sequence after its step
        _commit("commit_single", 1, 4, 8, 128, "4x2x2", 64, 512),
        # a batch after its step, all layers of a model
        _commit("commit_batch", 16, 32, 8, 128, "4x2x2x1x1", 64, 4000),
        # a decode round of a small batch: a page here and there
        _pages("pages_decode", 16, 64, 0, 4096),
        # a large batch with prompts that come in and requests that are done
        _pages("pages_prompts", 1024, 64, 512, 2048),
        # one sequence, penalties only, logits straight from a bf16 head, odd vocabulary
        _logits("logits_single", 1, "4x2x2", 50001, "bf16", 700, 0.0, 0),
        # the rows of a batched step (c4) under grammars, with penalties and biases
        _logits("logits_batch", 16, "4x2x2x1x1", 32000, "fp32", 4096, 0.02, 64),
    ]


TREES = ("1", "1x1x1x1", "2x2", "4x2x2", "8x2x1x1", "4x2x2x1x1", "4x4x2x1", "16", "3x3x3x2", "128")


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _bounded(make, *most):
    """A case made by `make` whose work is at most the most of the cases `most`."""
    limits = [work(c) for c in most]
    while True:
        case = make()
        w = work(case)
        if all(w[k] <= max(limit[k] for limit in limits) for k in ("bytes", "flops")):
            return case


def _unnamed(case):
    return {k: v for k, v in case.items() if k != "name"}


def draw(rng):
    kind = rng.choice(("attn", "attn", "rows", "commit", "pages", "logits"))
    by_name = {c["name"]: c for c in listed()}

    def attn():
        H_kv = rng.choice((1, 2, 4, 5, 8, 12, 32))
        hi = _log(rng, 1, 16384)
        return _unnamed(_attn("", _log(rng, 1, 32), H_kv * rng.choice((1, 1, 2, 4, 7, 8)), H_kv, rng.choice((32, 64, 96, 128, 128, 256)),
                              rng.choice((hi, max(1, hi // 16), 1)), hi, rng.choice(TREES), rng.choice((32, 64, 96, 128, 256))))

    def rows():
        return _unnamed(_rows("", _log(rng, 1, 16384), rng.choice((1, 2, 5, 8, 32)), rng.choice((32, 64, 96, 128, 256)),
                              rng.choice(("bf16", "fp32")), rng.choice((32, 64, 96, 256)), rng.random() < 0.5))

    def commit():
        return _unnamed(_commit("", _log(rng, 1, 32), _log(rng, 1, 32), rng.choice((1, 4, 8, 32)), rng.choice((64, 96, 128, 256)),
                                rng.choice(TREES[2:9]), rng.choice((32, 64, 128)), _log(rng, 1, 4000)))

    def pages():
        return _unnamed(_pages("", _log(rng, 1, 1024), rng.choice((32, 64, 96, 256)), rng.choice((0, _log(rng, 1, 512))), _log(rng, 1, 8192)))

    def logits():
        return _unnamed(_logits("", _log(rng, 1, 32), rng.choice(TREES), rng.choice((_log(rng, 64, 65536), 32000, 50001, 65536)),
                                rng.choice(("bf16", "fp32")), _log(rng, 1, 16384), rng.choice((0.0, 0.001, 0.5, 0.99)), rng.choice((0, 7, 300))))

    if kind == "attn":
        return _bounded(attn, by_name["attn_tree_long"], by_name["attn_tree_batch"])
    if kind == "rows":
        return _bounded(rows, by_name["rows_prompts"])
    if kind == "commit":
        return _bounded(commit, by_name["commit_batch"])
    if kind == "pages":
        return pages()
    return _bounded(logits, by_name["logits_batch"])


def tree_of(text):
    """Parent array (generation order, -1 = child of the root) and depths of a k-configuration."""
    parent, depth, level = [], [], [-1]
    for n, k in enumerate(int(x) for x in text.split("x")):
        nxt = []
        for p in level:
            for _ in range(k):
                nxt.append(len(parent))
                parent.append(p)
                depth.append(n + 1)
        level = nxt
    return parent, depth


def lengths(case):
    """Prefix lengths of a batch: spread over [lo, hi], the longest first, in a fixed order."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    return [hi - int(math.floor((hi - lo) * ((b * 0.6180339887498949) % 1.0))) for b in range(B)]


def work(case):
    kind = case["kind"]
    if kind == "attn":
        parent, depth = tree_of(case["tree"])
        N, d, H_q, H_kv, B = len(parent), case["d"], case["H_q"], case["H_kv"], case["B"]
        total = sum(lengths(case))
        cache = 2 * H_kv * (d // 2 + d // 32) * total
        return {"bytes": cache + B * N * d * 2 * (2 * H_kv + 2 * H_q), "flops": 4 * d * H_q * (N * total + B * sum(depth))}
    if kind == "rows":
        values = 2 * case["T"] * case["H_kv"] * case["d"]
        packed = values // 2 + values // 32
        return {"bytes": 2 * (values * (4 if case["dtype"] == "fp32" else 2) + packed), "flops": 4 * values}
    if kind == "commit":
        _, depth = tree_of(case["tree"])
        rows = sum(1 + _accepted(b, max(depth)) for b in range(case["B"])) * case["layers"]
        values = 2 * rows * case["H_kv"] * case["d"]
        return {"bytes": 2 * (values * 2 + values // 2 + values // 32), "flops": 4 * values}
    if kind == "pages":
        _, prefix, want, max_pages, slots = _requests(case)
        held = sum(-(-n // case["page"]) for n in prefix)
        need = sum(-(-n // case["page"]) for n in want)
        return {"bytes": 4 * (6 * case["B"] + 4 * abs(need - held) + 2 * slots), "flops": 4 * slots + 8 * case["B"]}
    N, V, B = len(tree_of(case["tree"])[0]), case["V"], case["B"]
    per_value = (2 if case["dtype"] == "bf16" else 4) + 4 + (0.125 if case["mask"] else 0)
    return {"bytes": int(B * (1 + N) * V * per_value + 4 * B * case["hist"]), "flops": 4 * B * (1 + N) * V}


# ---------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def encode_plain(x):
    """Codes uint8 [..., d / 32, 16] and scales uint8 [..., d / 32] of rows [..., d]."""
    d = x.shape[-1]
    x = x.float().reshape(*x.shape[:-1], d // BLOCK, BLOCK)
    amax = x.abs().amax(-1)
    bad = ~torch.isfinite(amax)
    mantissa, exponent = torch.frexp(torch.where(bad, torch.ones_like(amax), amax))
    e = torch.where(mantissa <= 0.875, exponent - 3, exponent - 2)          # 7 * 2^e = 0.875 * 2^(e + 3) holds the largest
    e = torch.where(amax == 0, torch.full_like(e, -119), e).clamp(-119, 125)
    y = torch.ldexp(x, -e.unsqueeze(-1))
    a = y.abs()
    code = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int()
    code = (code + 8 * torch.signbit(y).int()) * (~bad).unsqueeze(-1)
    scale = torch.where(bad, torch.full_like(e, 255), e + 127)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), scale.to(torch.uint8)


def decode_plain(codes, scales):
    """Rows fp32 [..., d] of codes [..., d / 32, 16] and scales [..., d / 32]."""
    both = torch.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], BLOCK).long()
    table = torch.tensor(CODE_VALUES + tuple(-v for v in CODE_VALUES), dtype=torch.float32, device=codes.device)
    s = scales.int()
    values = torch.ldexp(table[both], (s - 127).unsqueeze(-1))
    values = torch.where((s == 255).unsqueeze(-1), torch.full_like(values, float("nan")), values)
    return values.reshape(*codes.shape[:-2], codes.shape[-2] * BLOCK)


def _empty_pool(n_pages, H_kv, page, d, lead=()):
    shape = (*lead, n_pages, H_kv, page // TILE, d // BLOCK, TILE)
    return torch.zeros(*shape, 16, dtype=torch.uint8, device=DEV), torch.full(shape, 127, dtype=torch.uint8, device=DEV)


def _prepare_attn(case, seed):
    g = _generator(seed)
    B, H_q, H_kv, d, page = (case[k] for k in ("B", "H_q", "H_kv", "d", "page"))
    parent, _ = tree_of(case["tree"])
    N, lens = len(parent), lengths(case)
    max_pages = -(-case["hi"] // page)
    n_pages = sum(-(-n // page) for n in lens) + 3
    order = torch.randperm(n_pages, generator=g, device=DEV).int()
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(lens):
        k = -(-n // page)
        table[b, :k] = order[at:at + k]
        at += k
    pools = []
    for _ in range(2):
        codes, scales = _empty_pool(n_pages, H_kv, page, d)
        for p0 in range(0, n_pages, 256):               # a part at a time: the values in 32 bits are eight times the codes
            n = min(256, n_pages - p0)
            x = torch.randn(n, H_kv, page // TILE, TILE, d, generator=g, device=DEV)
            c, s = encode_plain(x)
            codes[p0:p0 + n] = c.transpose(3, 4)
            scales[p0:p0 + n] = s.transpose(3, 4)
        pools += [codes, scales]
    normal = lambda *shape: torch.randn(*shape, generator=g, device=DEV).bfloat16()
    st = {"case": case, "lens": lens, "table": table, "pools": pools, "q": normal(B, N, H_q, d), "k_tree": normal(B, H_kv, N, d),
          "v_tree": normal(B, H_kv, N, d), "parent": _ints(parent), "prefix_len": _ints(lens), "scale": 1.0 / math.sqrt(d)}
    mask = torch.zeros(N, N, dtype=torch.bool)
    for i in range(N):
        a = i
        while a >= 0:
            mask[i, a] = True
            a = parent[a]
    st["mask"] = mask.to(DEV)
    if own:
        from paper_2401_06706_amd import binding as M
        st["out"] = torch.empty_like(st["q"])
        kv = M.fourbit_kv(*pools, block_table=table)
        args = M.fourbit_attn_args(st["q"], kv, st["prefix_len"], st["k_tree"], st["v_tree"], st["parent"], st["out"], st["scale"], case["hi"])
        need = M.mcsd_attn_fourbit_workspace_bytes(args.desc)
        st["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
        st["args"] = M.fourbit_attn_args(st["q"], kv, st["prefix_len"], st["k_tree"], st["v_tree"], st["parent"], st["out"], st["scale"],
                                         case["hi"], st["workspace"])
    return st


def _prepare_rows(case, seed):
    g = _generator(seed)
    T, H_kv, d, page = (case[k] for k in ("T", "H_kv", "d", "page"))
    dtype = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    n_pages = -(-T // page) + 2
    # channels of different size, as keys have them
    spread = torch.exp(torch.randn(H_kv, d, generator=g, device=DEV))
    if case["fused"]:
        both = torch.randn(T, 2, H_kv, d, generator=g, device=DEV).mul_(spread).to(dtype)
        k, v = both[:, 0], both[:, 1]
    else:
        k = torch.randn(T, H_kv, d, generator=g, device=DEV).mul_(spread).to(dtype)
        v = torch.randn(T, H_kv, d, generator=g, device=DEV).to(dtype)
    order = torch.randperm(n_pages, generator=g, device=DEV)
    pos = torch.arange(T, device=DEV)
    slots = (order[pos // page] * page + pos % page).int()
    k_codes, k_scales = _empty_pool(n_pages, H_kv, page, d)
    v_codes, v_scales = _empty_pool(n_pages, H_kv, page, d)
    st = {"case": case, "k": k, "v": v, "slots": slots, "pools": [k_codes, k_scales, v_codes, v_scales],
          "k_back": torch.empty(T, H_kv, d, dtype=dtype, device=DEV), "v_back": torch.empty(T, H_kv, d, dtype=dtype, device=DEV)}
    if own:
        from paper_2401_06706_amd import binding as M
        kv = M.fourbit_kv(*st["pools"])
        st["store"] = M.fourbit_rows_args(k, v, slots, kv)
        st["load"] = M.fourbit_rows_args(st["k_back"], st["v_back"], slots, kv)
    return st


def _accepted(b, gamma):
    return (3 * b + 2) % (gamma + 1)


def _prepare_commit(case, seed):
    g = _generator(seed)
    B, layers, H_kv, d, page, L = (case[k] for k in ("B", "layers", "H_kv", "d", "page", "L"))
    parent, depth = tree_of(case["tree"])
    N, gamma = len(parent), max(depth)
    capacity = L + gamma + 1
    max_pages = -(-capacity // page)
    n_pages = B * max_pages + 2
    table = torch.randperm(n_pages, generator=g, device=DEV)[:B * max_pages].reshape(B, max_pages).int()
    lens = [max(0, L - 7 * b) for b in range(B)]
    leaves = [i for i in range(N) if depth[i] == gamma]
    pick = torch.randint(0, len(leaves), (B,), generator=g, device=DEV).tolist()
    n_accepted, paths = [], []
    for b in range(B):
        path, a = [], leaves[pick[b]]
        while a >= 0:
            path.insert(0, a)
            a = parent[a]
        n = _accepted(b, gamma)
        n_accepted.append(n)
        paths.append(path[:n] + [-1] * (gamma - n))
    host_table = table.tolist()
    slots = []
    for b in range(B):
        for j in range(gamma + 1):
            r = lens[b] + j
            slots.append(host_table[b][r // page] * page + r % page if j <= n_accepted[b] else -1)
    pools = []
    for _ in range(2):
        pools += list(_empty_pool(n_pages, H_kv, page, d, (layers,)))
    normal = lambda: torch.randn(layers, B, H_kv, 1 + N, d, generator=g, device=DEV).bfloat16()
    i32 = dict(dtype=torch.int32, device=DEV)
    back = lambda: torch.zeros(layers, B * (gamma + 1), H_kv, d, dtype=torch.bfloat16, device=DEV)
    st = {"case": case, "pools": pools, "k_tree": normal(), "v_tree": normal(), "start": _ints(lens), "prefix_len": _ints(lens),
          "n_accepted": _ints(n_accepted), "path": _ints(paths), "table": table, "slots": _ints(slots),
          "tokens": torch.randint(0, 32000, (B, gamma + 1), generator=g, **i32), "next_root": torch.zeros(B, **i32),
          "flags": torch.zeros(B, **i32), "k_back": back(), "v_back": back()}
    if own:
        from paper_2401_06706_amd import binding as M
        kv = M.fourbit_kv(*pools, block_table=table)
        st["args"] = M.fourbit_commit_args(kv, st["k_tree"], st["v_tree"], st["n_accepted"], st["path"], st["tokens"], st["prefix_len"],
                                           st["next_root"], st["flags"], capacity, root_row=True)
        st["load"] = M.fourbit_rows_args(st["k_back"], st["v_back"], st["slots"], kv)
    return st


def _requests(case):
    """Lengths now and wanted of every request: most go on by a tree's depth, every ninth is done, and with prompts every
    fourth is new.  Returns B, lengths, wanted lengths, table width and the slots wanted."""
    B, live = case["B"], case["live"]
    prefix, want = [], []
    for b in range(B):
        n = 1 + int(live * ((b * 0.6180339887498949 + 0.25) % 1.0))
        if case["prompt"] and b % 4 == 1:
            prefix.append(0)
            want.append(1 + int(case["prompt"] * ((b * 0.4142135623730951 + 0.5) % 1.0)))
        elif b % 9 == 5:
            prefix.append(n)
            want.append(0)
        else:
            prefix.append(n)
            want.append(n + 6)
    slots = sum(max(0, w - p) for p, w in zip(prefix, want))
    max_pages = -(-(max(max(prefix), max(want))) // case["page"])
    return B, prefix, want, max_pages, slots


def _prepare_pages(case, seed):
    g = _generator(seed)
    page = case["page"]
    B, prefix, want, max_pages, slots = _requests(case)
    held = [-(-n // page) for n in prefix]
    need = [-(-n // page) for n in want]
    # room for nearly all: the last sequences of a full pool have to wait
    n_pages = sum(held) + sum(max(0, b - a) for a, b in zip(held, need)) - sum(max(0, a - b) for a, b in zip(held, need))
    n_pages = max(n_pages - B // 64, sum(held), 1) + 1
    order = torch.randperm(n_pages, generator=g, device=DEV).int()
    sizes = [B, 1, n_pages, B * max_pages]
    pristine = torch.full((sum(sizes),), -1, dtype=torch.int32, device=DEV)

    def parts(t):
        a, b, c, d = torch.split(t, sizes)
        return {"held": a, "n_free": b, "free": c, "table": d.view(B, max_pages)}
    p = parts(pristine)
    p["held"].copy_(_ints(held))
    p["n_free"].fill_(n_pages - sum(held))
    p["free"][:n_pages - sum(held)] = order[sum(held):]
    at = 0
    for b in range(B):
        p["table"][b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    state = torch.empty_like(pristine)
    st = {"case": case, "pristine": pristine, "state": state, **parts(state), "prefix_len": _ints(prefix), "want_len": _ints(want),
          "slots": slots, "flags": torch.zeros(B, dtype=torch.int32, device=DEV),
          "slot_start": torch.zeros(B + 1, dtype=torch.int32, device=DEV), "slot_map": torch.zeros(slots + 5, dtype=torch.int32, device=DEV)}
    if own:
        from paper_2401_06706_amd import binding as M
        st["args"] = M.page_args(st["prefix_len"], st["want_len"], st["held"], st["table"], st["free"], st["n_free"], st["flags"],
                                 page, st["slot_start"], st["slot_map"])
    return st


def _prepare_logits(case, seed):
    g = _generator(seed)
    B, V, H = case["B"], case["V"], case["hist"]
    parent, _ = tree_of(case["tree"])
    N = len(parent)
    dtype = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    skewed = lambda *shape: (V * torch.rand(*shape, generator=g, device=DEV) ** 3).int().clamp_(max=V - 1)
    hist_len = [max(1, H - int(0.5 * H * ((b * 0.6180339887498949) % 1.0))) for b in range(B)]
    u = lambda lo, hi: lo + (hi - lo) * torch.rand(B, generator=g, device=DEV)
    st = {"case": case, "logits": (3.0 * torch.randn(B, 1 + N, V, generator=g, device=DEV)).to(dtype),
          "out": torch.empty(B, 1 + N, V, dtype=torch.float32, device=DEV), "parent": _ints(parent), "host_parent": parent,
          "cand": skewed(B, N), "history": skewed(B, H), "hist_len": _ints(hist_len), "prompt_len": _ints([n // 2 for n in hist_len]),
          "repetition": u(1.0, 1.3), "presence": u(0.0, 0.5), "frequency": u(0.0, 0.3), "bias_tok": None, "bias_val": None, "mask": None}
    if case["bias"]:
        n = min(case["bias"], V)
        st["bias_tok"] = torch.stack([torch.randperm(V, generator=g, device=DEV)[:n] for _ in range(B)]).int()
        st["bias_val"] = 4.0 * torch.randn(B, n, generator=g, device=DEV)
    if case["mask"]:
        words = -(-V // 32)
        bits = torch.rand(B, 1 + N, words * 32, generator=g, device=DEV) < case["mask"]
        bits[:, :, V // 2] = True                       # a grammar always lets something through
        free = torch.rand(B, 1 + N, 1, generator=g, device=DEV) < 0.25
        bits |= free                                    # rows inside free text
        st["mask"] = _pack_bits(bits)
    if own:
        from paper_2401_06706_amd import binding as M
        st["args"] = M.logits_args(st["logits"], st["out"], st["parent"], st["cand"], st["history"], st["hist_len"], st["prompt_len"],
                                   st["repetition"], st["presence"], st["frequency"], st["bias_tok"], st["bias_val"], st["mask"])
    return st


def _pack_bits(bits):
    weights = (1 << torch.arange(32, dtype=torch.int64, device=DEV))
    words = torch.empty(*bits.shape[:-1], bits.shape[-1] // 32, dtype=torch.int32, device=DEV)
    for b in range(bits.shape[0]):                      # (a sequence at a time: 64 bits per bit)
        w = (bits[b].reshape(bits.shape[1], -1, 32).long() * weights).sum(-1)
        words[b] = torch.where(w >= 2 ** 31, w - 2 ** 32, w).int()
    return words


def prepare(case, seed):
    return {"attn": _prepare_attn, "rows": _prepare_rows, "commit": _prepare_commit, "pages": _prepare_pages,
            "logits": _prepare_logits}[case["kind"]](case, seed)


# ---------------------------------------------------------------------------- one pass
def _pool_rows(codes, scales, pages):
    """Rows fp32 [H_kv][len(pages) * page size][d] of the pages named."""
    c, s = codes[pages], scales[pages]                              # [P][H_kv][tiles][d/32][16][16]
    rows = decode_plain(c.transpose(3, 4), s.transpose(3, 4))       # [P][H_kv][tiles][16][d]
    P, H_kv, tiles, _, d = rows.shape
    return rows.permute(1, 0, 2, 3, 4).reshape(H_kv, P * tiles * TILE, d)


def _run_attn(st):
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_tree_attn_fourbit(st["args"])
        return st["out"]
    case, q = st["case"], st["q"]
    B, N, H_q, d = q.shape
    H_kv, page = case["H_kv"], case["page"]
    G = H_q // H_kv
    out = torch.empty_like(q)
    for b, L in enumerate(st["lens"]):
        pages = st["table"][b, :-(-L // page)].long()
        k = torch.cat((_pool_rows(st["pools"][0], st["pools"][1], pages)[:, :L], st["k_tree"][b].float()), 1)
        v = torch.cat((_pool_rows(st["pools"][2], st["pools"][3], pages)[:, :L], st["v_tree"][b].float()), 1)
        qb = q[b].float().reshape(N, H_kv, G, d).permute(1, 0, 2, 3).reshape(H_kv, N * G, d)
        s = torch.matmul(qb, k.transpose(1, 2).contiguous()) * st["scale"]
        s[:, :, L:].masked_fill_(~st["mask"].repeat_interleave(G, 0), float("-inf"))
        e = torch.exp(s - s.amax(-1, keepdim=True))
        o = torch.matmul(e, v) / e.sum(-1, keepdim=True)
        out[b] = o.reshape(H_kv, N, G, d).permute(1, 0, 2, 3).reshape(N, H_q, d).to(q.dtype)
    return out


def _places(slots, page):
    s = slots.long()
    return s // page, s % page // TILE, s % TILE


def _store_plain(pool, x, slots, page):
    codes, scales = encode_plain(x)                                 # [T][H_kv][d/32][16], [T][H_kv][d/32]
    p, t, r = _places(slots, page)
    pool[0][p, :, t, :, r] = codes
    pool[1][p, :, t, :, r] = scales


def _load_plain(pool, slots, page):
    p, t, r = _places(slots, page)
    return decode_plain(pool[0][p, :, t, :, r], pool[1][p, :, t, :, r])


def _run_rows(st):
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_kv_store_fourbit(st["store"])
        M.mcsd_kv_load_fourbit(st["load"])
        return st["k_back"], st["v_back"]
    page, slots = st["case"]["page"], st["slots"]
    back = []
    for i, x in ((0, st["k"]), (2, st["v"])):
        pool = st["pools"][i:i + 2]
        _store_plain(pool, x, slots, page)
        back.append(_load_plain(pool, slots, page).to(x.dtype))
    return tuple(back)


def _run_commit(st):
    st["prefix_len"].copy_(st["start"])
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_kv_commit_fourbit(st["args"])
        M.mcsd_kv_load_fourbit(st["load"])
        return st["k_back"], st["v_back"], st["prefix_len"], st["next_root"], st["flags"]
    page, layers = st["case"]["page"], st["case"]["layers"]
    B, gamma = st["path"].shape
    n = st["n_accepted"].long()
    j = torch.arange(gamma + 1, device=DEV)
    take = j.unsqueeze(0) <= n.unsqueeze(1)                         # the root, then the path
    source = torch.cat((torch.zeros(B, 1, dtype=torch.long, device=DEV), st["path"].long() + 1), 1)
    b_of, j_of = take.nonzero(as_tuple=True)
    pos = st["prefix_len"].long()[b_of] + j_of
    slots = st["table"][b_of, pos // page].long() * page + pos % page
    at = b_of * (gamma + 1) + j_of
    for layer in range(layers):
        for i, tree, back in ((0, st["k_tree"], st["k_back"]), (2, st["v_tree"], st["v_back"])):
            pool = [st["pools"][i][layer], st["pools"][i + 1][layer]]
            _store_plain(pool, tree[layer][b_of, :, source[b_of, j_of]], slots, page)
            back[layer][at] = _load_plain(pool, slots, page).to(back.dtype)
    st["prefix_len"] += 1 + st["n_accepted"]
    st["next_root"].copy_(st["tokens"].gather(1, n.unsqueeze(1)).squeeze(1))
    st["flags"].zero_()
    return st["k_back"], st["v_back"], st["prefix_len"], st["next_root"], st["flags"]


def _run_pages(st):
    st["state"].copy_(st["pristine"])
    outputs = tuple(st[k] for k in ("table", "held", "free", "n_free", "flags", "slot_start", "slot_map"))
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_page_assign(st["args"])
        return outputs
    page, table, held, free = st["case"]["page"], st["table"], st["held"], st["free"]
    B, width = table.shape
    col = torch.arange(width, device=DEV)
    need = (st["want_len"] + page - 1) // page
    # pages that are no longer needed go back, the first of them on top
    surplus = (held - need).clamp(min=0)
    before = torch.cumsum(surplus, 0) - surplus
    total = st["n_free"] + surplus.sum()
    back = (col >= need.unsqueeze(1)) & (col < held.unsqueeze(1))
    b_of, c_of = back.nonzero(as_tuple=True)
    free[(total - 1 - (before[b_of] + c_of - need[b_of])).long()] = table[b_of, c_of]
    table[b_of, c_of] = -1
    # in order, as long as they last
    lack = (need - held).clamp(min=0)
    upto = torch.cumsum(lack, 0)
    served = (lack == 0) | (upto <= total)
    give = lack * served
    fresh = served.unsqueeze(1) & (col >= held.unsqueeze(1)) & (col < need.unsqueeze(1))
    b_of, c_of = fresh.nonzero(as_tuple=True)
    table[b_of, c_of] = free[(total - 1 - ((upto - lack)[b_of] + c_of - held[b_of])).long()]
    held.copy_(torch.where(served, need, held))
    st["n_free"].copy_(total - give.sum())
    st["flags"].copy_(torch.where(served, 0, 256))
    # a slot for every new token
    count = torch.where(served, (st["want_len"] - st["prefix_len"]).clamp(min=0), 0)
    st["slot_start"][0] = 0
    st["slot_start"][1:] = torch.cumsum(count, 0)
    slot_map = st["slot_map"]
    i = torch.arange(slot_map.numel(), device=DEV)
    b_of = torch.searchsorted(st["slot_start"][1:].contiguous(), i.int(), right=True)
    inside = b_of < B
    b_of = b_of.clamp(max=B - 1)
    pos = torch.where(inside, st["prefix_len"][b_of] + i - st["slot_start"][b_of], 0)
    slot_map.copy_(torch.where(inside, table[b_of, pos // page].long() * page + pos % page, -1))
    return outputs


def _run_logits(st):
    if own:
        from paper_2401_06706_amd import binding as M
        M.mcsd_logits_rules(st["args"])
        return st["out"]
    B, rows, V = st["logits"].shape
    N, parent = rows - 1, st["host_parent"]
    pos = torch.arange(st["history"].shape[1], device=DEV)
    live = pos < st["hist_len"].unsqueeze(1)
    after = live & (pos >= st["prompt_len"].unsqueeze(1))
    for b in range(B):
        tokens = st["history"][b].long()
        seen = torch.zeros(V, device=DEV).index_add_(0, tokens, live[b].float())
        count = torch.zeros(rows, V, device=DEV)
        count[0] = torch.zeros(V, device=DEV).index_add_(0, tokens, after[b].float())
        for i in range(N):
            count[1 + i] = count[1 + parent[i]]
            count[1 + i].index_add_(0, st["cand"][b, i:i + 1].long(), torch.ones(1, device=DEV))
        z = st["logits"][b].float()
        r = st["repetition"][b]
        z = torch.where((seen > 0) | (count > 0), torch.where(z > 0, z / r, z * r), z)
        z = z - st["frequency"][b] * count - st["presence"][b] * (count > 0)
        if st["bias_tok"] is not None:
            z = z + torch.zeros(V, device=DEV).index_put_((st["bias_tok"][b].long(),), st["bias_val"][b])
        if st["mask"] is not None:
            word = st["mask"][b].repeat_interleave(32, 1)[:, :V]
            bit = (word >> (torch.arange(V, device=DEV, dtype=torch.int32) % 32)) & 1
            z = z.masked_fill(bit == 0, float("-inf"))
        st["out"][b] = z
    return st["out"]


def run(state):
    return {"attn": _run_attn, "rows": _run_rows, "commit": _run_commit, "pages": _run_pages, "logits": _run_logits}[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------- from the definitions, in 64 bits
def _value64(code):
    """e2m1: sign, two exponent bits (bias 1), one mantissa bit."""
    c = code.to(torch.int64)
    exponent, mantissa = (c >> 1) & 3, (c & 1).double()
    magnitude = torch.where(exponent == 0, 0.5 * mantissa, (1.0 + 0.5 * mantissa) * torch.pow(2.0, (exponent - 1).double()))
    return torch.where((c & 8) != 0, -magnitude, magnitude)


def _page64(codes, scales):
    """[H_kv][page size][d] of one page."""
    H_kv, tiles, blocks, rows, _ = codes.shape
    out = torch.empty(H_kv, tiles, rows, blocks, BLOCK, dtype=torch.float64, device=codes.device)
    factor = torch.pow(2.0, scales.double() - 127.0).permute(0, 1, 3, 2)
    c = codes.permute(0, 1, 3, 2, 4)
    out[..., 0::2] = _value64(c % 16) * factor.unsqueeze(-1)
    out[..., 1::2] = _value64(c // 16) * factor.unsqueeze(-1)
    return out.reshape(H_kv, tiles * rows, blocks * BLOCK)


def _nearest64(x):
    """What rows [..., d] stand for once they are held in 4 bits, in 64 bits."""
    shape = x.shape
    x = x.double().reshape(-1, BLOCK)
    largest = x.abs().max(1).values
    e = torch.full_like(largest, 125.0)
    while True:                                             # the smallest power whose sevenfold holds the largest value
        lower = (largest <= 7.0 * torch.pow(2.0, e - 1.0)) & (e > -119.0)
        if not bool(lower.any()):
            break
        e = torch.where(lower, e - 1.0, e)
    y = x / torch.pow(2.0, e).unsqueeze(1)
    best, best_distance = torch.zeros_like(y), y.abs()
    for code in (2, 4, 6, 1, 3, 5, 7):                      # even codes first: they keep ties
        v = CODE_VALUES[code]
        near = (y.abs() - v).abs()
        closer = near < best_distance
        best = torch.where(closer, torch.full_like(best, v), best)
        best_distance = torch.minimum(best_distance, near)
    return (torch.where(y < 0, -best, best) * torch.pow(2.0, e).unsqueeze(1)).reshape(shape)


def _exact_attn(st):
    case, q = st["case"], st["q"]
    B, N, H_q, d = q.shape
    G, page = H_q // case["H_kv"], case["page"]
    out = torch.empty(q.shape, dtype=torch.float64, device=DEV)
    for b in range(B):
        L = st["lens"][b]
        ks, vs = [], []
        for i in range(-(-L // page)):
            p = int(st["table"][b, i])
            ks.append(_page64(st["pools"][0][p], st["pools"][1][p]))
            vs.append(_page64(st["pools"][2][p], st["pools"][3][p]))
        k, v = torch.cat(ks, 1), torch.cat(vs, 1)
        for g in range(case["H_kv"]):
            kg = torch.cat((k[g, :L], st["k_tree"][b, g].double()))
            vg = torch.cat((v[g, :L], st["v_tree"][b, g].double()))
            hidden = torch.zeros(N, L + N, dtype=torch.bool, device=DEV)
            hidden[:, L:] = ~st["mask"]
            for h in range(g * G, (g + 1) * G):
                s = (q[b, :, h].double() @ kg.t()) * st["scale"]
                s[hidden] = float("-inf")
                out[b, :, h] = torch.softmax(s, -1) @ vg
    return out


def _exact_commit(st):
    B, gamma = st["path"].shape
    tokens, paths, n = st["tokens"].tolist(), st["path"].tolist(), st["n_accepted"].tolist()
    back = []
    for tree in (st["k_tree"], st["v_tree"]):
        rows = torch.zeros(st["case"]["layers"], B * (gamma + 1), tree.shape[2], tree.shape[4], dtype=torch.float64, device=DEV)
        for b in range(B):
            for j in range(1 + n[b]):
                rows[:, b * (gamma + 1) + j] = _nearest64(tree[:, b, :, 0 if j == 0 else 1 + paths[b][j - 1]])
        back.append(rows)
    start = st["start"].tolist()
    return (*back, _ints([start[b] + 1 + n[b] for b in range(B)]), _ints([tokens[b][n[b]] for b in range(B)]), _ints([0] * B))


def _exact_pages(st):
    page = st["case"]["page"]
    st["state"].copy_(st["pristine"])
    table, held, free, n_free = st["table"].tolist(), st["held"].tolist(), st["free"].tolist(), int(st["n_free"])
    prefix, want = st["prefix_len"].tolist(), st["want_len"].tolist()
    B = len(prefix)
    need = [-(-w // page) for w in want]
    for b in range(B - 1, -1, -1):                          # the last page back lies on top: sequence 0's first surplus one
        for c in range(held[b] - 1, need[b] - 1, -1):
            free[n_free], table[b][c] = table[b][c], -1
            n_free += 1
    held = [min(h, n) for h, n in zip(held, need)]
    flags, asked, top, starts, slots = [], 0, n_free, [0], []
    for b in range(B):
        lack = need[b] - held[b]
        asked += lack
        fits = lack == 0 or asked <= top
        flags.append(0 if fits else 256)
        if fits:
            for c in range(held[b], need[b]):
                n_free -= 1
                table[b][c] = free[n_free]
            held[b] = need[b]
            slots += [table[b][i // page] * page + i % page for i in range(prefix[b], want[b])]
        starts.append(len(slots))
    slots += [-1] * (st["slot_map"].numel() - len(slots))
    return tuple(_ints(x) for x in (table, held, free, [n_free], flags, starts, slots))


def _exact_logits(st):
    B, rows, V = st["logits"].shape
    out = torch.empty(B, rows, V, dtype=torch.float64, device=DEV)
    parent = st["host_parent"]
    for b in range(B):
        n, first = int(st["hist_len"][b]), int(st["prompt_len"][b])
        base = torch.bincount(st["history"][b, first:n].long(), minlength=V)
        prompt = torch.bincount(st["history"][b, :first].long(), minlength=V) > 0
        r, f, p = (float(st[k][b]) for k in ("repetition", "frequency", "presence"))
        cand = st["cand"][b].tolist()
        for row in range(rows):
            count, a = base.clone(), row - 1
            while a >= 0:
                count[cand[a]] += 1
                a = parent[a]
            z = st["logits"][b, row].double()
            used = prompt | (count > 0)
            z[used] = torch.where(z[used] > 0, z[used] / r, z[used] * r)
            z -= f * count.double() + p * (count > 0).double()
            if st["bias_tok"] is not None:
                z[st["bias_tok"][b].long()] += st["bias_val"][b].double()
            if st["mask"] is not None:
                words = st["mask"][b, row].long() & 0xFFFFFFFF
                allowed = ((words.unsqueeze(1) >> torch.arange(32, device=DEV)) & 1).bool().reshape(-1)[:V]
                z[~allowed] = float("-inf")
            out[b, row] = z
    return out


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "attn":
        return _exact_attn(st)
    if kind == "rows":
        return _nearest64(st["k"]), _nearest64(st["v"])
    if kind == "commit":
        return _exact_commit(st)
    if kind == "pages":
        return _exact_pages(st)
    return _exact_logits(st)
