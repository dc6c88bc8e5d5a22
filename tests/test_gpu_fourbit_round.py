"""Decode rounds with a paged cache held in 4 bits, as they are used together and without a host read in between: pages from the
lengths, prompts stored by slot, tree attention of every layer, rules on the logits, verification, commit, pages again; against the same rounds in
plain steps, eagerly and as one captured graph that is replayed."""
import numpy as np
import pytest
import torch

from oracle import mcsd_oracle as O
from paper_2401_06706_amd import binding as M
from paper_2401_06706_amd import workloads as W
from tests import fourbit_ref as F
from tests.test_gpu_fourbit import DEV, dev_bf16, f64, i32
from tests.test_gpu_logits_rules import pack
from tests.test_gpu_pages import account

pytestmark = pytest.mark.gpu


class Loop:
    """B sequences, LAYERS layers; every round's model outputs (queries, tree keys and values, logits, candidates) are fresh inputs."""
    B, LAYERS, H_q, H_kv, d, ps, V, kconfig = 3, 2, 4, 2, 64, 32, 500, (3, 2)

    def __init__(self, seed=0):
        self.rng = np.random.default_rng(seed)
        self.N, _ = M.mcsd_tree_size(self.kconfig)
        self.gamma = len(self.kconfig)
        self.width, self.n_pages = 6, 16
        self.prompts = [40, 1, 63]
        self.tokens = self.rng.integers(0, self.V, size=(self.B, 200)).astype(np.int32)      # history buffer
        B, N, g = self.B, self.N, self.gamma
        z = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
        self.t = dict(prefix=z(B), want=z(B), held=z(B), table=torch.full((B, self.width), -1, dtype=torch.int32, device=DEV),
                      free=i32(self.rng.permutation(self.n_pages)), n_free=i32([self.n_pages]), page_flags=z(B), start=z(B + 1), slots=z(128),
                      parent=z(N), depth=z(N), q_row=z(1 + N), hist=i32(self.tokens), hist_len=z(B), prompt_len=z(B), cand=z(B, N),
                      n_acc=z(B), path=z(B, g), out_tok=z(B, g + 1), acc_child=z(B, 1 + N), endpoint=z(B, 1 + N), vflags=z(B, 1 + N), next_root=z(B), cflags=z(B))
        cs, ss = M.fourbit_shapes(self.n_pages, self.H_kv, self.ps, self.d, self.LAYERS)
        self.pools = [torch.full(s, v, dtype=torch.uint8, device=DEV) for s, v in ((cs, 0x3c), (ss, 255), (cs, 0x3c), (ss, 255))]
        self.cache = M.fourbit_kv(*self.pools, block_table=self.t["table"])
        self.layer = [M.fourbit_kv(*[p[l] for p in self.pools], block_table=self.t["table"]) for l in range(self.LAYERS)]
        M.mcsd_tree_build(self.kconfig, self.t["parent"], self.t["depth"], self.t["q_row"])
        rows = 1 + N
        bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)
        f = lambda *s: torch.zeros(*s, device=DEV)
        self.x = dict(k_prompt=bf(self.LAYERS, 128, self.H_kv, self.d), v_prompt=bf(self.LAYERS, 128, self.H_kv, self.d), q=bf(self.LAYERS, B, rows, self.H_q, self.d),
                      k_tree=bf(self.LAYERS, B, self.H_kv, rows, self.d), v_tree=bf(self.LAYERS, B, self.H_kv, rows, self.d), out=bf(self.LAYERS, B, rows, self.H_q, self.d),
                      target=f(B, rows, self.V), ruled=f(B, rows, self.V), draft=f(B, 4, self.V), u_acc=f(B, N), u_end=f(B, rows), temp=torch.ones(B, device=DEV),
                      rep=f(B), pres=f(B), freq=f(B), mask=torch.zeros(B, rows, (self.V + 31) // 32, dtype=torch.int32, device=DEV))
        t, x = self.t, self.x
        self.pages = M.page_args(t["prefix"], t["want"], t["held"], t["table"], t["free"], t["n_free"], t["page_flags"], self.ps, t["start"], t["slots"])
        self.store = M.fourbit_rows_args(x["k_prompt"], x["v_prompt"], t["slots"], self.cache)
        L = self.width * self.ps
        make = lambda l, ws: M.fourbit_attn_args(x["q"][l], self.layer[l], t["prefix"], x["k_tree"][l], x["v_tree"][l], t["parent"], x["out"][l], self.d ** -0.5, L, ws)
        need = M.mcsd_attn_fourbit_workspace_bytes(make(0, None).desc)
        self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
        self.attn = [make(l, self.ws) for l in range(self.LAYERS)]
        self.rules = M.logits_args(x["target"], x["ruled"], t["parent"], t["cand"], t["hist"], t["hist_len"], t["prompt_len"], x["rep"], x["pres"], x["freq"], mask=x["mask"])
        self.verify = M.verify_args(x["ruled"], x["draft"], t["q_row"], t["parent"], t["cand"], x["u_acc"], x["u_end"], x["temp"], t["n_acc"], t["path"], t["out_tok"],
                                    t["acc_child"], t["endpoint"], t["vflags"], M.WITH_REPLACEMENT)
        self.commit = M.fourbit_commit_args(self.cache, x["k_tree"], x["v_tree"], t["n_acc"], t["path"], t["out_tok"], t["prefix"], t["next_root"], t["cflags"], L, root_row=True)

    def start(self):
        self.t["want"].copy_(i32(self.prompts))
        for k in ("k_prompt", "v_prompt"):
            self.x[k].copy_(dev_bf16(self.rng, *self.x[k].shape))
        M.mcsd_page_assign(self.pages)
        M.mcsd_kv_store_fourbit(self.store)
        self.t["prefix"].copy_(self.t["want"])
        self.t["hist_len"].copy_(self.t["want"])
        self.t["prompt_len"].copy_(self.t["want"])

    def feed(self):
        """What the models would bring to the next round."""
        x, B, N, V = self.x, self.B, self.N, self.V
        for k in ("q", "k_tree", "v_tree"):
            x[k].copy_(dev_bf16(self.rng, *x[k].shape))
        target = (2 * self.rng.normal(size=(B, 1 + N, V))).astype(np.float32)
        x["target"].copy_(torch.from_numpy(target))
        x["draft"].copy_(torch.from_numpy((2 * self.rng.normal(size=(B, 4, V))).astype(np.float32)))
        self.mask = self.rng.random((B, 1 + N, V)) < 0.5
        cand = self.rng.integers(0, V, size=(B, N)).astype(np.int32)
        self.mask[np.arange(B)[:, None], 1 + np.arange(N)[None], cand] = True
        x["mask"].copy_(torch.from_numpy(pack(self.mask)))
        self.t["cand"].copy_(torch.from_numpy(cand))
        u = lambda *s: torch.from_numpy((self.rng.integers(1, 2 ** 24, size=s) / 2.0 ** 24).astype(np.float32))
        x["u_acc"].copy_(0.02 * u(B, N))
        x["u_end"].copy_(u(B, 1 + N))
        x["rep"].fill_(1.25); x["pres"].fill_(0.5); x["freq"].fill_(0.25)

    def round(self):
        t = self.t
        torch.add(t["prefix"], 1 + self.gamma, out=t["want"])
        M.mcsd_page_assign(self.pages)
        for a in self.attn:
            M.mcsd_tree_attn_fourbit(a)
        M.mcsd_logits_rules(self.rules)
        M.mcsd_verify_sample(self.verify)
        M.mcsd_kv_commit_fourbit(self.commit)


def host(t):
    return t.detach().cpu().numpy().copy()


def check_round(lp, before):
    """The round just run, from the state before it."""
    t, x = {k: host(v) for k, v in lp.t.items()}, lp.x
    want = before["prefix"] + 1 + lp.gamma
    ref = account(before["prefix"], want, before["held"], before["table"], before["free"], before["n_free"][0], lp.ps, lp.n_pages, 128)
    for k, name in (("table", "table"), ("held", "held"), ("n_free", "n_free"), ("flags", "page_flags"), ("slots", "slots"), ("start", "start")):
        assert (t[name] == ref[k]).all(), name
    assert (ref["flags"] == 0).all()
    # what every sequence held, kept by this test in full precision as well
    parent = t["parent"]
    vis = F.ancestors(np.r_[-1, np.where(parent < 0, 0, parent + 1)])
    for l in range(lp.LAYERS):
        for b in range(lp.B):
            k, v = (np.concatenate([F.decode(*F.encode(r)) for r in lp.rows[b][i][l]]).reshape(-1, lp.H_kv, lp.d).transpose(1, 0, 2) for i in (0, 1))
            assert k.shape[1] == before["prefix"][b]
            o, bound = F.attention(f64(x["q"][l, b]), k, v, f64(x["k_tree"][l, b]), f64(x["v_tree"][l, b]), vis, lp.d ** -0.5)
            assert (np.abs(f64(x["out"][l, b]) - o) <= bound).all()
    # rules: the values themselves are tested elsewhere; masked places here, and that verification saw the ruled rows
    ruled = host(x["ruled"])
    assert (np.isneginf(ruled) == ~lp.mask).all()
    orc = O.verify(ruled, host(x["draft"]), t["q_row"], parent, t["cand"], host(x["u_acc"]), host(x["u_end"]), host(x["temp"]), W.WITH_REPLACEMENT, gamma_max=lp.gamma, n_threads=4)
    near = (orc.margin < 1e-6).any(axis=1)
    n_acc = t["n_acc"]
    for b in range(lp.B):
        if near[b]:
            continue
        assert n_acc[b] == orc.n_accepted[b] and (t["path"][b] == orc.accepted_path[b]).all() and (t["out_tok"][b] == orc.out_tokens[b]).all()
        emitted = t["out_tok"][b][:n_acc[b] + 1]
        rows = [0] + [1 + c for c in t["path"][b][:n_acc[b]]]
        assert all(lp.mask[b, r, tok] for r, tok in zip(rows, emitted)), "only tokens that the grammar allows"
    assert (t["cflags"] == 0).all() and (t["prefix"] == before["prefix"] + 1 + n_acc).all()
    for b in range(lp.B):
        taken = [0] + [1 + c for c in t["path"][b][:n_acc[b]]]
        for i, name in ((0, "k_tree"), (1, "v_tree")):
            for l in range(lp.LAYERS):
                for r in taken:
                    lp.rows[b][i][l].append(f64(x[name][l, b, :, r]))
    return n_acc


def begin(lp):
    lp.start()
    torch.cuda.synchronize()
    slots = host(lp.t["slots"])
    assert (slots[:104] >= 0).all() and (slots[104:] == -1).all()
    lp.rows, at = [], 0
    for n in lp.prompts:
        lp.rows.append([[[f64(lp.x[k][l, at + j]) for j in range(n)] for l in range(lp.LAYERS)] for k in ("k_prompt", "v_prompt")])
        at += n


def test_rounds_one_after_the_other():
    lp = Loop()
    begin(lp)
    accepted = 0
    for _ in range(6):
        lp.feed()
        before = {k: host(v) for k, v in lp.t.items()}
        lp.round()
        torch.cuda.synchronize()
        accepted += int(check_round(lp, before).sum())
    assert accepted > 0, "the case must commit paths, not roots alone"
    # and everything goes back
    lp.t["want"].zero_()
    M.mcsd_page_assign(lp.pages)
    assert int(lp.t["n_free"]) == lp.n_pages and (host(lp.t["table"]) == -1).all()
    assert sorted(host(lp.t["free"]).tolist()) == list(range(lp.n_pages))


def test_rounds_as_a_replayed_graph_beside_eager_ones():
    lp, other = Loop(seed=1), Loop(seed=2)
    begin(lp)
    begin(other)
    lp.feed()
    # (the first call of every kernel outside the capture)
    saved = {k: v.clone() for k, v in lp.t.items()}
    pools = [p.clone() for p in lp.pools]
    lp.round()
    torch.cuda.synchronize()
    for k, v in saved.items():
        lp.t[k].copy_(v)
    for p, q in zip(lp.pools, pools):
        p.copy_(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lp.round()
    for _ in range(4):
        lp.feed()
        other.feed()
        before = {k: host(v) for k, v in lp.t.items()}
        before_other = {k: host(v) for k, v in other.t.items()}
        graph.replay()
        other.round()
        torch.cuda.synchronize()
        check_round(lp, before)
        check_round(other, before_other)
