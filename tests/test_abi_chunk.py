"""The C ABI of chunk attention, weight sums, eviction and token log probabilities without a GPU: struct layouts, and every argument error
by return code before anything touches the device (the pointers here are never dereferenced)."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2401_06706_amd import binding as M

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PTR = 4096


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(M.LIB_PATH):
        from paper_2401_06706_amd.build import build
        build(verbose=False)
    return M.lib()


def test_struct_layout_matches_header(tmp_path):
    structs = {"mcsd_store_bufs": M.StoreBufs, "mcsd_chunk_desc": M.ChunkDesc, "mcsd_chunk_bufs": M.ChunkBufs, "mcsd_sums_bufs": M.SumsBufs,
               "mcsd_evict_desc": M.EvictDesc, "mcsd_evict_bufs": M.EvictBufs, "mcsd_logprob_desc": M.LogprobDesc, "mcsd_logprob_bufs": M.LogprobBufs}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "mcsd.h"', "int main(void){"]
    for cname, ct in structs.items():
        lines.append(f'printf("{cname} %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname}.{f} %zu\\n", offsetof({cname}, {f}));' for f, _ in ct._fields_]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = {k: int(v) for k, v in (l.split() for l in subprocess.check_output([str(exe)], text=True).splitlines())}
    for cname, ct in structs.items():
        assert got[cname] == C.sizeof(ct)
        for f, _ in ct._fields_:
            assert got[f"{cname}.{f}"] == getattr(ct, f).offset, f


def make(ct, defaults, kw):
    a = {"struct_size": C.sizeof(ct), **defaults, **kw}
    assert set(a) <= {f for f, _ in ct._fields_}
    return ct(**a)


def refused(lib, name, calls, changes):
    """Every change of one struct's fields is refused with its code and a message; NULL structs too."""
    f = getattr(lib, name)
    ref = lambda s: None if s is None else C.byref(s)
    for i, kw, code in changes:
        ct, defaults = calls[i]
        structs = [make(c, d, {}) for c, d in calls]
        structs[i] = make(ct, defaults, kw)
        assert f(*[ref(s) for s in structs], None) == code, (name, kw)
        assert len(lib.mcsd_last_error()) > 0
    for i in range(len(calls)):
        structs = [make(c, d, {}) for c, d in calls]
        structs[i] = None
        assert f(*[ref(s) for s in structs], None) == -1, (name, i)
        for size in (0, C.sizeof(calls[i][0]) + 4):
            structs[i] = make(*calls[i], {"struct_size": size})
            assert f(*[ref(s) for s in structs], None) == -2, (name, i)


PAGED = dict(page_size=64, n_pages=200, max_pages_per_seq=64, block_table=PTR)
BAD_PAGED = [(dict(page_size=0), -2), (dict(page_size=16), -2), (dict(page_size=48), -2), (dict(n_pages=0), -2), (dict(n_pages=2 ** 26), -3)]
BAD_TABLE = BAD_PAGED + [(dict(block_table=None), -1), (dict(max_pages_per_seq=0), -2), (dict(max_pages_per_seq=63), -2)]


def test_store_refusals(lib):
    desc = dict(T=8, H_kv=2, d=128, dtype=M.DTYPE_BF16, n_layers=2, k_stride=256, v_stride=256, k_layer_stride=2048, v_layer_stride=2048)
    bufs = dict(k=PTR, v=PTR, slot_map=PTR, k_pool=PTR, v_pool=PTR)
    refused(lib, "mcsd_kv_store_paged", [(M.RowsDesc, desc), (M.StoreBufs, bufs), (M.PagedKV, PAGED)],
            [(0, kw, c) for kw, c in [(dict(T=-1), -2), (dict(H_kv=0), -2), (dict(n_layers=0), -2), (dict(dtype=2), -3), (dict(d=0), -3), (dict(d=260), -3),
                                      (dict(d=12), -3), (dict(k_stride=255), -2), (dict(v_stride=248), -2), (dict(k_stride=260), -2), (dict(T=2 ** 30 + 1), -3),
                                      (dict(n_layers=65536), -3), (dict(k_layer_stride=4), -2), (dict(v_layer_stride=-8), -2), (dict(H_kv=65536), -3),
                                      (dict(T=2 ** 27, k_stride=2 ** 40), -3)]] +
            [(1, kw, c) for kw, c in [(dict(k=None), -1), (dict(v=None), -1), (dict(slot_map=None), -1), (dict(k_pool=None), -1), (dict(v_pool=None), -1),
                                      (dict(k=PTR + 8), -2), (dict(v_pool=PTR + 2), -2)]] + [(2, kw, c) for kw, c in BAD_PAGED])
    nothing = [make(M.RowsDesc, desc, dict(T=0)), make(M.StoreBufs, {}, {}), make(M.PagedKV, PAGED, dict(block_table=None, max_pages_per_seq=0))]
    assert lib.mcsd_kv_store_paged(*[C.byref(s) for s in nothing], None) == 0


CHUNK = dict(B=2, T=40, H_q=4, H_kv=2, d=128, dtype=M.DTYPE_BF16, L_stride=4096, scale=0.1, q_stride=512)
BAD_CHUNK = [(dict(B=0), -2), (dict(T=-1), -2), (dict(H_q=0), -2), (dict(H_kv=0), -2), (dict(H_q=5), -2), (dict(L_stride=0), -2), (dict(L_stride=2 ** 22 + 1), -3),
             (dict(B=65536), -3), (dict(H_kv=65536, H_q=65536, q_stride=2 ** 24), -3), (dict(T=2 ** 28), -3), (dict(scale=-1.0), -2), (dict(scale=float("nan")), -2),
             (dict(scale=float("inf")), -2), (dict(d=264), -3), (dict(d=12), -3), (dict(dtype=7), -3), (dict(q_stride=504), -2), (dict(q_stride=516), -2)]


def test_chunk_refusals(lib):
    good = make(M.ChunkDesc, CHUNK, {})
    need = M.mcsd_chunk_workspace_bytes(good)
    assert need > 0 and need % 256 == 0
    for kw, _ in BAD_CHUNK:
        assert M.mcsd_chunk_workspace_bytes(make(M.ChunkDesc, CHUNK, kw)) == 0, kw
    assert M.mcsd_chunk_workspace_bytes(make(M.ChunkDesc, CHUNK, dict(L_stride=64))) == 0          # few keys are never cut
    bufs = dict(q=PTR, k_pool=PTR, v_pool=PTR, chunk_start=PTR, prefix_len=PTR, out=PTR, lse=None, workspace=PTR, workspace_bytes=need)
    refused(lib, "mcsd_chunk_attn_paged", [(M.ChunkDesc, CHUNK), (M.ChunkBufs, bufs), (M.PagedKV, PAGED)],
            [(0, kw, c) for kw, c in BAD_CHUNK] +
            [(1, kw, c) for kw, c in [(dict(q=None), -1), (dict(k_pool=None), -1), (dict(v_pool=None), -1), (dict(chunk_start=None), -1), (dict(prefix_len=None), -1),
                                      (dict(out=None), -1), (dict(workspace=None), -5), (dict(workspace_bytes=need - 1), -5), (dict(workspace=PTR + 64), -5),
                                      (dict(q=PTR + 8), -2), (dict(out=PTR + 4), -2), (dict(v_pool=PTR + 2), -2)]] + [(2, kw, c) for kw, c in BAD_TABLE])


def test_sums_refusals(lib):
    bufs = dict(last_rows=0, q=PTR, k_pool=PTR, chunk_start=PTR, prefix_len=PTR, lse=PTR, sums=PTR)
    refused(lib, "mcsd_attn_weight_sums", [(M.ChunkDesc, CHUNK), (M.SumsBufs, bufs), (M.PagedKV, PAGED)],
            [(0, kw, c) for kw, c in BAD_CHUNK] +
            [(1, kw, c) for kw, c in [(dict(q=None), -1), (dict(k_pool=None), -1), (dict(chunk_start=None), -1), (dict(prefix_len=None), -1), (dict(lse=None), -1),
                                      (dict(sums=None), -1), (dict(last_rows=-1), -2), (dict(q=PTR + 8), -2), (dict(k_pool=PTR + 4), -2)]] +
            [(2, kw, c) for kw, c in BAD_TABLE])


def test_evict_refusals(lib):
    desc = dict(B=2, H_kv=2, d=128, dtype=M.DTYPE_BF16, L_stride=4096, n_layers=1, n_first=4, n_recent=64)
    bufs = dict(k_pool=PTR, v_pool=PTR, sums=PTR, prefix_len=PTR, keep_len=PTR, out_table=None, kept=PTR, flags=PTR)
    refused(lib, "mcsd_kv_evict_paged", [(M.EvictDesc, desc), (M.EvictBufs, bufs), (M.PagedKV, PAGED)],
            [(0, kw, c) for kw, c in [(dict(B=0), -2), (dict(H_kv=0), -2), (dict(L_stride=0), -2), (dict(n_layers=0), -2), (dict(n_first=-1), -2), (dict(n_recent=-1), -2),
                                      (dict(d=4), -3), (dict(d=512), -3), (dict(dtype=-1), -3), (dict(B=65536), -3), (dict(L_stride=2 ** 22 + 1), -3),
                                      (dict(n_layers=2 ** 22), -3), (dict(n_layers=2 ** 31 - 1, H_kv=2 ** 31 - 1, B=65535), -3)]] +
            [(1, kw, c) for kw, c in [(dict(k_pool=None), -1), (dict(v_pool=None), -1), (dict(sums=None), -1), (dict(prefix_len=None), -1), (dict(keep_len=None), -1),
                                      (dict(kept=None), -1), (dict(flags=None), -1), (dict(k_pool=PTR + 8), -2), (dict(out_table=PTR), -2)]] +
            [(2, kw, c) for kw, c in BAD_TABLE])


def test_logprob_refusals(lib):
    desc = dict(rows=4, R=4, V=1000, dtype=M.DTYPE_FP32, n_top=5, row_stride=1000)
    bad = [(dict(rows=-1), -2), (dict(R=0), -2), (dict(V=0), -2), (dict(n_top=-1), -2), (dict(n_top=65), -3), (dict(V=4, n_top=5), -3), (dict(V=2 ** 30 + 1), -3),
           (dict(rows=2 ** 22 + 1), -3), (dict(dtype=3), -3), (dict(row_stride=999), -2)]
    bufs = dict(logits=PTR, row_map=PTR, tokens=PTR, temperature=None, logprob=PTR, entropy=None, rank=None, top_tok=PTR, top_logprob=PTR, flags=PTR, workspace=PTR,
                workspace_bytes=M.mcsd_logprob_workspace_bytes(make(M.LogprobDesc, desc, {})))
    for kw, _ in bad:
        assert M.mcsd_logprob_workspace_bytes(make(M.LogprobDesc, desc, kw)) == 0
    refused(lib, "mcsd_token_logprobs", [(M.LogprobDesc, desc), (M.LogprobBufs, bufs)], [(0, kw, c) for kw, c in bad] +
            [(1, kw, c) for kw, c in [(dict(logits=None), -1), (dict(tokens=None), -1), (dict(logprob=None), -1), (dict(flags=None), -1), (dict(top_tok=None), -1),
                                      (dict(top_logprob=None), -1), (dict(logits=PTR + 2), -2)]])
    five = make(M.LogprobDesc, desc, dict(rows=5))
    assert lib.mcsd_token_logprobs(C.byref(five), C.byref(make(M.LogprobBufs, bufs, dict(row_map=None))), None) == -2
    assert lib.mcsd_token_logprobs(C.byref(make(M.LogprobDesc, desc, dict(rows=0))), C.byref(make(M.LogprobBufs, {}, {})), None) == 0


def test_binding_refuses_what_is_not_on_a_gpu():
    import torch
    t = torch.zeros(4, 2, 64)
    pool = torch.zeros(3, 2, 32, 64)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    with pytest.raises(ValueError):
        M.store_args(t, t, i32(4), pool, pool)
    with pytest.raises(ValueError):
        M.chunk_attn_args(t, pool, pool, i32(1, 2), i32(2), i32(1), t, 0.1, 64)
    with pytest.raises(ValueError):
        M.weight_sums_args(t, pool, i32(1, 2), i32(2), i32(1), torch.zeros(4, 2), torch.zeros(1, 2, 64), 0.1)
    with pytest.raises(ValueError):
        M.evict_args(pool, pool, i32(1, 2), torch.zeros(1, 2, 64), i32(1), i32(1), i32(1, 2, 64), i32(1), 0, 0)
    with pytest.raises(ValueError):
        M.logprob_args(torch.zeros(2, 9), i32(2), torch.zeros(2), None, None, None, None, i32(2))
    # shapes that do not fit each other
    with pytest.raises(ValueError):
        M.chunk_attn_args(t, pool, pool[:, :1], i32(1, 2), i32(2), i32(1), t, 0.1, 64)
    with pytest.raises(ValueError):
        M.chunk_attn_args(t.bfloat16(), pool, pool, i32(1, 2), i32(2), i32(1), t, 0.1, 64)
    with pytest.raises(ValueError):
        M.logprob_desc(torch.zeros(9, 2).t(), i32(2))


def test_chunk_sizes_that_always_fit(lib):
    """T H_q / 32 + min(T, B) H_kv up to 2^23 has a plan, whatever the type, the head dimension and the capacity; far beyond there may be none."""
    for B, T, H_q, H_kv in [(1, 2 ** 23, 31, 31), (65535, 65535, 64, 64), (2 ** 15, 2 ** 15, 248, 248), (8, 2 ** 18, 1016, 8), (4, 2 ** 13, 32000, 1), (1, 1, 65535, 65535), (65535, 2 ** 20, 120, 60)]:
        assert T * H_q / 32 + min(T, B) * H_kv <= 2 ** 23 and T * H_q < 2 ** 30
        for d in (64, 128, 256):
            for dtype in (M.DTYPE_FP32, M.DTYPE_BF16):
                for cap in (65536, 2 ** 22):
                    assert M.mcsd_chunk_workspace_bytes(make(M.ChunkDesc, CHUNK, dict(B=B, T=T, H_q=H_q, H_kv=H_kv, d=d, dtype=dtype, L_stride=cap, q_stride=H_q * d))) > 0
    assert M.mcsd_chunk_workspace_bytes(make(M.ChunkDesc, CHUNK, dict(B=65535, T=17000, H_q=60000, H_kv=60000, q_stride=60000 * 128))) == 0


def test_logprob_workspace(lib):
    """Few long rows need one; it is asked for and checked."""
    desc = dict(rows=2, R=4, V=262144, dtype=M.DTYPE_FP32, n_top=5, row_stride=262144)
    need = M.mcsd_logprob_workspace_bytes(make(M.LogprobDesc, desc, {}))
    assert need > 0
    for kw in (dict(rows=129, R=200), dict(V=51199), dict(dtype=M.DTYPE_BF16, V=102399), dict(rows=0)):
        assert M.mcsd_logprob_workspace_bytes(make(M.LogprobDesc, desc, kw)) == 0, kw
    bufs = dict(logits=PTR, tokens=PTR, logprob=PTR, top_tok=PTR, top_logprob=PTR, flags=PTR, workspace=PTR, workspace_bytes=need)
    for kw in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=PTR + 128)):
        assert lib.mcsd_token_logprobs(C.byref(make(M.LogprobDesc, desc, {})), C.byref(make(M.LogprobBufs, bufs, kw)), None) == -5, kw
