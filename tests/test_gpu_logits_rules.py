"""Penalties, biases and masks on logit rows of candidate trees, against the same rules in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2401_06706_amd import binding as M

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).to(DEV)


def i32(a):
    return dev(np.asarray(a, np.int32))


def random_tree(rng, n):
    return np.array([rng.integers(-1, i) if i else -1 for i in range(n)], np.int32)


def reference(c):
    """out float64 [B][R][V] (NaN where no row goes) and the bound on rounding: every one of at most five operations in fp32 is off by half
    a step, 2^-24 of what it leaves, and what they leave is at most |z| R' + F count + P + |bias| with R' = max(R, 1/R)."""
    z = c["logits"].astype(np.float64)
    B, R, V = z.shape
    out, bound = np.full(z.shape, np.nan), np.zeros(z.shape)
    N = c["cand"].shape[1]
    for b in range(B):
        parent = c["parent"][b] if c["parent"].ndim == 2 else c["parent"]
        rmap = np.arange(1 + N) if c["row_map"] is None else (c["row_map"][b] if c["row_map"].ndim == 2 else c["row_map"])
        hist = c["history"][b, :max(0, min(c["hist_len"][b], c["history"].shape[1]))]
        pl = 0 if c["prompt_len"] is None else c["prompt_len"][b]
        rep, pres, freq = (float(c[k][b]) if c[k] is not None else v for k, v in (("repetition", 1.0), ("presence", 0.0), ("frequency", 0.0)))
        bias = np.zeros(V)
        if c["bias_tok"] is not None:
            for t, v in zip(c["bias_tok"][b], c["bias_val"][b]):
                if 0 <= t < V:
                    bias[t] = v
        for r in range(*c["rows"]):
            row = rmap[r]
            if not 0 <= row < R:
                continue
            path, a = [], r - 1
            while a >= 0:
                path.append(c["cand"][b, a])
                a = parent[a]
            count, seen = np.zeros(V), np.zeros(V, bool)
            for i, t in enumerate(list(hist) + path):
                if 0 <= t < V:
                    seen[t] = True
                    if i >= len(hist) or i >= pl:
                        count[t] += 1
            with np.errstate(invalid="ignore", over="ignore"):
                y = np.where(seen, np.where(z[b, row] > 0, z[b, row] / rep, z[b, row] * rep), z[b, row])
                y = y - freq * count - pres * (count > 0) + bias
                bound[b, row] = 5 * 2.0 ** -24 * (np.abs(z[b, row]) * max(rep, 1 / rep) + abs(freq) * count + abs(pres) + np.abs(bias))
            if c["mask"] is not None:
                y[~c["mask"][b, row]] = -np.inf
            out[b, row] = y
    return out, bound


def pack(mask):
    B, R, V = mask.shape
    W = (V + 31) // 32
    bits = np.zeros((B, R, W * 32), np.uint64)
    bits[..., :V] = mask
    bits[..., V:] = np.random.default_rng(V).integers(0, 2, size=(B, R, W * 32 - V))      # bits behind the vocabulary mean nothing
    return (bits.reshape(B, R, W, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)


def make(B, V, N, S, seed=0, dtype="fp32", n_bias=0, allow=None, per_seq=False, row_map=None, R=None, rows=None, chain=False, none=()):
    rng = np.random.default_rng(seed)
    parent = np.arange(-1, N - 1, dtype=np.int32) if chain else random_tree(rng, N)
    if per_seq:
        parent = np.stack([random_tree(rng, N) for _ in range(B)])
    R = R or 1 + N
    tok = lambda *s: (V * rng.random(s) ** 3).astype(np.int32)
    c = dict(parent=parent, cand=tok(B, N), history=tok(B, S), row_map=row_map, rows=rows or (0, 1 + N))
    c["hist_len"] = rng.integers(0, S + 1, size=B).astype(np.int32)
    if B > 1:
        c["hist_len"][0], c["hist_len"][1] = S, 0
    c["prompt_len"] = (c["hist_len"] // 2).astype(np.int32)
    c["repetition"] = rng.uniform(0.7, 1.5, size=B).astype(np.float32)
    c["presence"], c["frequency"] = rng.uniform(-1, 1, size=B).astype(np.float32), rng.uniform(-0.3, 0.5, size=B).astype(np.float32)
    c["bias_tok"], c["bias_val"] = (rng.integers(-2, V + 2, size=(B, n_bias)).astype(np.int32), rng.normal(size=(B, n_bias)).astype(np.float32)) if n_bias else (None, None)
    if S > 2:
        c["history"][:, 0], c["history"][:, 1] = -1, V           # passed over
    c["mask"] = None if allow is None else rng.random((B, R, V)) < allow
    z = torch.from_numpy((3 * rng.normal(size=(B, R, V))).astype(np.float32))
    c["t"] = (z.bfloat16() if dtype == "bf16" else z).to(DEV)
    c["logits"] = c["t"].float().cpu().numpy()
    for k in none:
        c[k] = None
    return c


def args_of(c, logits, out):
    opt = lambda k, f=dev: None if c[k] is None else f(c[k])
    tree = c["cand"].shape[1] > 0
    hist = c["history"].shape[1] > 0
    return M.logits_args(logits, out, i32(c["parent"]) if tree else None, i32(c["cand"]) if tree else None, i32(c["history"]) if hist else None,
                         i32(c["hist_len"]) if hist else None, opt("prompt_len", i32), opt("repetition"), opt("presence"), opt("frequency"),
                         opt("bias_tok", i32), opt("bias_val"), None if c["mask"] is None else dev(pack(c["mask"])), opt("row_map", i32), c["rows"])


def check(c, inplace=False):
    out = c["t"].clone() if inplace else torch.full(c["t"].shape, 55.0, dtype=torch.float32, device=DEV)
    M.mcsd_logits_rules(args_of(c, out if inplace else c["t"], out))
    torch.cuda.synchronize()
    got = out.cpu().numpy().astype(np.float64)
    want, bound = reference(c)
    rest = np.isnan(want)
    was = c["logits"].astype(np.float64) if inplace else np.full(got.shape, 55.0)
    assert (got[rest] == was[rest]).all(), "rows that no tree row names are left alone"
    fin = np.isfinite(want)
    assert (got[~fin & ~rest] == want[~fin & ~rest]).all()
    err = np.abs(got - want)[fin]
    assert (err <= bound[fin]).all(), float((err - bound[fin]).max())
    return out


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("kw", [
    dict(B=1, V=1, N=0, S=1), dict(B=2, V=33, N=3, S=5, n_bias=3, allow=0.5), dict(B=2, V=1024, N=6, S=100, n_bias=40, allow=0.02),
    dict(B=3, V=1027, N=28, S=300, n_bias=7, allow=0.9), dict(B=2, V=4096, N=128, S=2000, chain=True, allow=0.3), dict(B=2, V=32000, N=12, S=4096, n_bias=300),
    dict(B=1, V=50001, N=5, S=700, allow=0.001), dict(B=70, V=300, N=2, S=64, n_bias=5), dict(B=2, V=130000, N=1, S=50, n_bias=9, allow=0.5),
    dict(B=3, V=2048, N=9, S=128, per_seq=True, allow=0.4), dict(B=2, V=512, N=5, S=0, n_bias=4), dict(B=2, V=512, N=5, S=40, none=("repetition", "frequency", "prompt_len")),
    dict(B=2, V=512, N=5, S=40, none=("presence",)), dict(B=2, V=640, N=6, S=90, rows=(2, 5), allow=0.5), dict(B=2, V=640, N=6, S=90, rows=(3, 3)),
], ids=lambda kw: "-".join(f"{k}{v}" for k, v in kw.items() if k != "none"))
def test_against_64_bits(kw, inplace):
    check(make(**kw), inplace)


@pytest.mark.parametrize("V", [64, 1023, 2052, 32000])
def test_bf16_logits(V):
    check(make(3, V, 7, 200, dtype="bf16", n_bias=5, allow=0.6))


@pytest.mark.parametrize("per_seq", [False, True])
def test_rows_by_map(per_seq):
    """The draft's rows: those with children, in another order, and rows that nothing names."""
    rmap = np.array([3, -1, 0, 9, -1, 1, 4], np.int32)
    if per_seq:
        rmap = np.stack([rmap, rmap[::-1], np.roll(rmap, 2)])
    check(make(3, 777, 6, 50, allow=0.5, row_map=rmap, R=6, per_seq=per_seq))


def test_values_that_are_no_numbers_and_rows_without_a_token():
    c = make(2, 300, 3, 80, allow=0.5, n_bias=4)
    c["t"][0, 0, :40], c["t"][0, 1, 5], c["t"][1, 2, 7] = float("-inf"), float("inf"), float("nan")
    c["bias_val"][0, :] = -np.inf
    c["mask"][0, 0, 60:] = True
    c["mask"][1, 3] = False
    c["logits"] = c["t"].cpu().numpy()
    out = torch.zeros(2, 4, 300, device=DEV)
    M.mcsd_logits_rules(args_of(c, c["t"], out))
    got = out.cpu().numpy()
    assert (got[1, 3] == -np.inf).all()
    assert (got[~c["mask"]] == -np.inf).all(), "a masked place is -infinity whatever stood there"
    want, _ = reference(c)
    assert np.isposinf(got[0, 1, 5]) == np.isposinf(want[0, 1, 5])
    assert (np.isnan(got) == np.isnan(want)).all() and (np.isneginf(got) == np.isneginf(want)).all()


def test_a_row_without_a_token_is_flagged_by_the_verification():
    """Masked logits go into the verification as they are; a row that has none left is flagged there and the others are as ever."""
    from paper_2401_06706_amd import device as D
    from paper_2401_06706_amd import workloads as W
    from tests.parity import run_oracle
    vi = W.gen_verify_inputs(W.WORKLOADS["c2"].with_(B=2, V=600, variant=W.WITH_REPLACEMENT))
    call = D.make_verify_call(vi)
    rows = 1 + vi.N
    mask = np.random.default_rng(0).random((2, rows, 600)) < 0.7
    np.put_along_axis(mask[:, 1:], vi.cand_tok[..., None].astype(np.int64), True, -1)
    mask[1, 0] = False
    z = call.tensors["target_logits"]
    M.mcsd_logits_rules(M.logits_args(z, z, call.tensors["parent"], call.tensors["cand_tok"], mask=dev(pack(mask))))
    M.mcsd_verify_sample(call.args)
    torch.cuda.synchronize()
    got = call.results()
    assert got["flags"][1, 0] & M.FLAG_NONFINITE and not (got["flags"][0] & M.FLAG_NONFINITE).any() and not (got["flags"][1, 1:] & M.FLAG_NONFINITE).any()
    vi.target_logits[:] = z.cpu().numpy()
    orc = run_oracle(vi)
    ok = orc.margin >= 1e-6
    ok[1, 0] = False
    assert (got["acc_child"] == orc.acc_child)[ok].all() and (got["endpoint"] == orc.endpoint)[ok].all()
    emitted = got["endpoint"][0]
    assert all(mask[0, r, t] for r, t in enumerate(emitted) if t >= 0)


def test_last_entry_of_a_token_counts():
    V, n = 100, 1000
    tok = np.random.default_rng(1).integers(0, V, size=(1, n)).astype(np.int32)
    val = np.arange(n, dtype=np.float32)[None]
    z = torch.zeros(1, 1, V, device=DEV)
    M.mcsd_logits_rules(M.logits_args(z, z, bias_tok=i32(tok), bias_val=dev(val)))
    want = np.zeros(V)
    want[tok[0]] = val[0]
    assert (z.cpu().numpy()[0, 0] == want).all()


@pytest.mark.parametrize("offset", [0, 1, 2, 3])
def test_rows_that_start_anywhere(offset):
    """Logits and results that start at any word, and results at another offset than the logits."""
    c = make(2, 1024, 4, 60, allow=0.5, n_bias=3)
    n = c["t"].numel()
    z, o = torch.empty(n + 4, device=DEV), torch.full((n + 8,), 4.0, device=DEV)
    z[offset:offset + n] = c["t"].flatten()
    k = (2 * offset + 1) % 4
    zi, oo = z[offset:offset + n].view(2, 5, 1024), o[k:k + n].view(2, 5, 1024)
    M.mcsd_logits_rules(args_of(c, zi, oo))
    want, bound = reference(c)
    got = oo.cpu().numpy().astype(np.float64)
    fin = np.isfinite(want)
    assert (got[~fin] == want[~fin]).all() and (np.abs(got - want)[fin] <= bound[fin]).all()
    assert (o[:k] == 4).all() and (o[k + n:] == 4).all()


def test_in_a_graph_beside_eager_calls():
    c = make(2, 5000, 8, 500, allow=0.5, n_bias=9)
    out = torch.zeros(2, 9, 5000, device=DEV)
    args = args_of(c, c["t"], out)
    M.mcsd_logits_rules(args)
    torch.cuda.synchronize()
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.mcsd_logits_rules(args)
    for _ in range(3):
        out.zero_()
        graph.replay()
        check(make(1, 900, 3, 40))
        assert torch.equal(out, want)
