"""The C ABI of the 4-bit cache, the pages and the logit rules without a GPU: struct layouts, and every argument error
by return code before anything touches the device (the pointers here are never dereferenced)."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2401_06706_amd import binding as M

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(M.LIB_PATH):
        from paper_2401_06706_amd.build import build
        build(verbose=False)
    return M.lib()


def test_struct_layout_matches_header(tmp_path):
    structs = {"mcsd_fourbit_kv": M.FourbitKV, "mcsd_rows_desc": M.RowsDesc, "mcsd_rows_bufs": M.RowsBufs, "mcsd_page_desc": M.PageDesc,
               "mcsd_page_bufs": M.PageBufs, "mcsd_logits_desc": M.LogitsDesc, "mcsd_logits_bufs": M.LogitsBufs}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "mcsd.h"', "int main(void){"]
    for cname, ct in structs.items():
        lines.append(f'printf("{cname} %zu\\n", sizeof({cname}));')
        lines += [f'printf("{cname}.{f} %zu\\n", offsetof({cname}, {f}));' for f, _ in ct._fields_]
    for name in ("CACHE_FULL", "BAD_PAGES", "SLOTS_FULL"):
        lines.append(f'printf("flag.{name} %d\\n", MCSD_FLAG_{name});')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0;}"]))
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = {k: int(v) for k, v in (l.split() for l in subprocess.check_output([str(exe)], text=True).splitlines())}
    for cname, ct in structs.items():
        assert got[cname] == C.sizeof(ct)
        for f, _ in ct._fields_:
            assert got[f"{cname}.{f}"] == getattr(ct, f).offset, f
    assert (got["flag.CACHE_FULL"], got["flag.BAD_PAGES"], got["flag.SLOTS_FULL"]) == (M.FLAG_CACHE_FULL, M.FLAG_BAD_PAGES, M.FLAG_SLOTS_FULL)


def kv(**kw):
    a = dict(size=C.sizeof(M.FourbitKV), page_size=64, n_pages=200, max_pages=64, table=4096, kc=4096, vc=4096, ks=4096, vs=4096)
    a.update(kw)
    return M.FourbitKV(*a.values())


BAD_KV = [(dict(size=8), -2), (dict(page_size=0), -2), (dict(page_size=16), -2), (dict(page_size=48), -2), (dict(n_pages=0), -2), (dict(kc=None), -1),
          (dict(vc=None), -1), (dict(ks=None), -1), (dict(vs=None), -1), (dict(kc=4104), -2), (dict(vs=4097), -2), (dict(n_pages=2 ** 26), -3)]


def attn_desc(**kw):
    a = dict(B=2, N=6, H_q=4, H_kv=2, d=128, dtype=M.DTYPE_BF16, L_stride=4096, scale=0.088)
    a.update(kw)
    return M.attn_desc(**a)


def test_attention_refusals(lib):
    d = attn_desc()
    need = M.mcsd_attn_fourbit_workspace_bytes(d)
    assert need > 0 and need % 256 == 0
    bufs = lambda **kw: M.AttnBufs(*{**dict(size=C.sizeof(M.AttnBufs), q=4096, kp=None, vp=None, len=4096, kt=4096, vt=4096, parent=4096, out=4096, ws=4096, n=need), **kw}.values())
    call = lambda d, b, k: lib.mcsd_tree_attn_fourbit(None if d is None else C.byref(d), None if b is None else C.byref(b), None if k is None else C.byref(k), None)
    for kw, code in [(dict(N=0), -4), (dict(N=129), -4), (dict(H_q=5), -2), (dict(B=0), -2), (dict(B=65536), -3), (dict(d=72), -3), (dict(d=288), -3),
                     (dict(dtype=M.DTYPE_FP32), -3), (dict(dtype=9), -3), (dict(scale=float("inf")), -2), (dict(scale=-1.0), -2), (dict(L_stride=-1), -2),
                     (dict(H_kv=70000, H_q=70000), -3), (dict(L_stride=1 << 23), -3)]:
        bad = attn_desc(**kw)
        assert M.mcsd_attn_fourbit_workspace_bytes(bad) == 0
        assert call(bad, bufs(), kv(max_pages=1 << 20)) == code, kw
        assert len(lib.mcsd_last_error()) > 0
    for kw, code in BAD_KV + [(dict(table=None), -1), (dict(max_pages=0), -2), (dict(max_pages=63), -2)]:
        assert call(d, bufs(), kv(**kw)) == code, kw
    for kw, code in [(dict(size=3), -2), (dict(q=None), -1), (dict(len=None), -1), (dict(kt=None), -1), (dict(vt=None), -1), (dict(parent=None), -1),
                     (dict(out=None), -1), (dict(ws=None), -5), (dict(n=need - 1), -5), (dict(ws=4096 + 64), -5), (dict(q=4104), -2), (dict(out=4100), -2)]:
        assert call(d, bufs(**kw), kv()) == code, kw
    assert call(None, bufs(), kv()) == -1 and call(d, None, kv()) == -1 and call(d, bufs(), None) == -1


def test_commit_refusals(lib):
    desc = lambda **kw: M.CommitDesc(C.sizeof(M.CommitDesc), *{**dict(B=2, N=6, H_kv=2, d=128, dtype=1, L_stride=64, gamma_max=2, n_layers=1, root_row=0), **kw}.values())
    ptrs = [None, None] + [4096] * 8
    bufs = lambda p=ptrs: M.CommitBufs(C.sizeof(M.CommitBufs), *p)
    call = lambda d, b, k: lib.mcsd_kv_commit_fourbit(C.byref(d), C.byref(b), None if k is None else C.byref(k), None)
    for kw, code in [(dict(N=0), -4), (dict(N=129), -4), (dict(B=0), -2), (dict(d=48), -3), (dict(d=40, dtype=0), -3), (dict(dtype=5), -3), (dict(L_stride=0), -2),
                     (dict(gamma_max=0), -2), (dict(n_layers=0), -2), (dict(root_row=2), -2), (dict(B=70000), -3)]:
        assert call(desc(**kw), bufs(), kv()) == code, kw
    for i in range(2, 10):
        assert call(desc(), bufs(ptrs[:i] + [None] + ptrs[i + 1:]), kv()) == -1, i
    for kw, code in BAD_KV + [(dict(table=None), -1), (dict(max_pages=0), -2)]:
        assert call(desc(), bufs(), kv(**kw)) == code, kw
    assert call(desc(), bufs(ptrs[:2] + [4104] + ptrs[3:]), kv()) == -2
    assert call(desc(), bufs(), None) == -1


@pytest.mark.parametrize("name", ["mcsd_kv_store_fourbit", "mcsd_kv_load_fourbit"])
def test_rows_refusals(lib, name):
    desc = lambda **kw: M.RowsDesc(C.sizeof(M.RowsDesc), *{**dict(T=5, H_kv=2, d=128, dtype=1, n_layers=1, ks=256, vs=256, kl=0, vl=0), **kw}.values())
    bufs = lambda **kw: M.RowsBufs(*{**dict(size=C.sizeof(M.RowsBufs), k=4096, v=4096, slots=4096), **kw}.values())
    call = lambda d, b, k: getattr(lib, name)(None if d is None else C.byref(d), None if b is None else C.byref(b), None if k is None else C.byref(k), None)
    for kw, code in [(dict(T=-1), -2), (dict(H_kv=0), -2), (dict(n_layers=0), -2), (dict(dtype=2), -3), (dict(d=16), -3), (dict(d=288), -3), (dict(d=100), -3),
                     (dict(ks=255), -2), (dict(vs=128), -2), (dict(ks=260), -2), (dict(dtype=0, ks=258), -2), (dict(n_layers=70000), -3), (dict(T=2 ** 30 + 1), -3), (dict(T=2 ** 27, H_kv=2, d=128), -3), (dict(T=2 ** 20, H_kv=1024, d=32, ks=2 ** 15, vs=2 ** 15), -3),
                     (dict(n_layers=2, kl=1283), -2), (dict(n_layers=2, vl=-1280), -2)]:
        assert call(desc(**kw), bufs(), kv(table=None)) == code, kw
    for kw, code in BAD_KV:
        assert call(desc(), bufs(), kv(**kw)) == code, kw
    for kw, code in [(dict(size=4), -2), (dict(k=None), -1), (dict(v=None), -1), (dict(slots=None), -1), (dict(k=4104), -2)]:
        assert call(desc(), bufs(**kw), kv()) == code, kw
    assert call(None, bufs(), kv()) == -1 and call(desc(), None, kv()) == -1 and call(desc(), bufs(), None) == -1
    assert call(desc(T=0), bufs(k=None), kv()) == 0


def test_page_refusals(lib):
    desc = lambda **kw: M.PageDesc(C.sizeof(M.PageDesc), *{**dict(B=2, page_size=64, n_pages=20, max_pages=4, max_slots=8), **kw}.values())
    names = [n for n, _ in M.PageBufs._fields_[1:]]
    bufs = lambda **kw: M.PageBufs(C.sizeof(M.PageBufs), *{**{n: 4096 for n in names}, **kw}.values())
    call = lambda d, b: lib.mcsd_page_assign(None if d is None else C.byref(d), None if b is None else C.byref(b), None)
    for kw, code in [(dict(B=0), -2), (dict(B=65536), -3), (dict(page_size=0), -2), (dict(n_pages=0), -2), (dict(max_pages=0), -2), (dict(max_slots=-1), -2), (dict(max_slots=2 ** 30 + 1), -3), (dict(max_slots=2 ** 31 - 1), -3),
                     (dict(n_pages=1 << 25), -3)]:
        assert call(desc(**kw), bufs()) == code, kw
    for n in names:
        assert call(desc(), bufs(**{n: None})) == -1, n
    assert call(desc(), bufs(slot_start=None, slot_map=None)) == -1           # slots wanted without a map
    d = desc()
    d.struct_size = 4
    assert call(d, bufs()) == -2 and call(None, bufs()) == -1 and call(desc(), None) == -1


def test_logits_refusals(lib):
    desc = lambda **kw: M.LogitsDesc(C.sizeof(M.LogitsDesc), *{**dict(B=2, N=6, V=1000, R=7, dtype=0, per_seq=0, begin=0, end=7, S=10, n_bias=2), **kw}.values())
    names = [n for n, _ in M.LogitsBufs._fields_[1:]]
    bufs = lambda **kw: M.LogitsBufs(C.sizeof(M.LogitsBufs), *{**{n: 1 << 20 for n in names}, "row_map": None, **kw}.values())
    call = lambda d, b: lib.mcsd_logits_rules(None if d is None else C.byref(d), None if b is None else C.byref(b), None)
    for kw, code in [(dict(B=0), -2), (dict(B=65536), -3), (dict(V=0), -2), (dict(V=2 ** 30 + 1), -3), (dict(N=-1), -4), (dict(N=129), -4), (dict(R=0), -2), (dict(R=6), -2),
                     (dict(dtype=2), -3), (dict(per_seq=2), -2), (dict(begin=-1), -2), (dict(begin=5, end=4), -2), (dict(end=8), -2), (dict(S=-1), -2), (dict(n_bias=-1), -2)]:
        assert call(desc(**kw), bufs()) == code, kw
    for n in ("logits", "out", "parent", "cand_tok", "history", "hist_len", "bias_tok", "bias_val"):
        assert call(desc(), bufs(**{n: None})) == -1, n
    # in place is the very same place; anything else must not overlap
    assert call(desc(), bufs(out=(1 << 20) + 64)) == -2 and call(desc(), bufs(out=(1 << 20) - 64)) == -2
    assert call(desc(dtype=1), bufs()) == -2                                   # bf16 logits can not become fp32 in place
    assert call(desc(), bufs(logits=(1 << 20) + 2, out=1 << 25)) == -2
    d = desc()
    d.struct_size = 4
    assert call(d, bufs()) == -2 and call(None, bufs()) == -1 and call(desc(), None) == -1
    assert call(desc(begin=3, end=3), bufs()) == 0                             # no rows, no work


def test_the_binding_refuses_what_is_not_on_a_gpu():
    u8 = lambda s: torch.zeros(s, dtype=torch.uint8)
    codes, scales = M.fourbit_shapes(2, 1, 32, 64)
    assert codes == (2, 1, 2, 2, 16, 16) and scales == (2, 1, 2, 2, 16)
    assert M.fourbit_shapes(2, 1, 32, 64, 3)[1] == (3, 2, 1, 2, 2, 16)
    for bad in ((u8(codes), u8(scales), u8(codes), u8(scales)), (u8(scales), u8(scales), u8(codes), u8(scales)), (u8(codes), u8(codes), u8(codes), u8(scales))):
        with pytest.raises(ValueError):
            M.fourbit_kv(*bad)
    z = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        M.page_args(z, z, z, torch.zeros(2, 3, dtype=torch.int32), z, z[:1], z, 32)
    with pytest.raises(ValueError):
        M.page_args(z, z, z, torch.zeros(2, 3, dtype=torch.int32), z, z[:1], z, 32, slot_map=z)
    x = torch.zeros(2, 1, 10)
    with pytest.raises(ValueError):
        M.logits_args(x, x)
    with pytest.raises(ValueError):
        M.logits_args(x, x, parent=z)
