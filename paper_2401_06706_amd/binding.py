"""ctypes binding of libmcsd.so: argument marshalling only.

Every function here fills the C structs of include/mcsd.h from torch tensors
(device pointers, shapes) and calls the entry point of the same name; all
computation happens in the HIP kernels.  There is no fallback: if the library
is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmcsd.so")

DTYPE_FP32, DTYPE_BF16 = 0, 1
WITH_REPLACEMENT, WITHOUT_REPLACEMENT, NAIVE = 0, 1, 2
MAX_NODES, MAX_VOCAB = 128, 65536

FLAG_NEAR_TIE_ACCEPT, FLAG_NEAR_TIE_ENDPOINT, FLAG_BAD_TOKEN = 1, 2, 4
FLAG_ZERO_DRAFT_PROB, FLAG_ZERO_RESIDUAL, FLAG_NONFINITE, FLAG_BAD_TREE = 8, 16, 32, 64
FLAG_CACHE_FULL, FLAG_BAD_PAGES, FLAG_SLOTS_FULL = 256, 512, 1024

EXPORTS = ["mcsd_last_error", "mcsd_version", "mcsd_tree_validate", "mcsd_attn_workspace_bytes",
           "mcsd_tree_attn", "mcsd_tree_attn_static", "mcsd_attn_plan_override", "mcsd_tree_attn_paged", "mcsd_verify_workspace_bytes", "mcsd_verify_sample", "mcsd_verify_step",
           "mcsd_draft_sample", "mcsd_tree_size", "mcsd_tree_build", "mcsd_kv_commit", "mcsd_kv_commit_paged",
           "mcsd_tree_attn_fourbit", "mcsd_attn_fourbit_workspace_bytes", "mcsd_kv_commit_fourbit",
           "mcsd_kv_store_fourbit", "mcsd_kv_load_fourbit", "mcsd_page_assign", "mcsd_logits_rules",
           "mcsd_kv_store_paged", "mcsd_chunk_workspace_bytes", "mcsd_chunk_attn_paged", "mcsd_attn_weight_sums", "mcsd_kv_evict_paged",
           "mcsd_logprob_workspace_bytes", "mcsd_token_logprobs",
           "mcsd_kernel_timing", "mcsd_kernel_count", "mcsd_kernel_name", "mcsd_kernel_timing_read"]


class McsdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libmcsd error {code}: {msg}")
        self.code = code


class AttnDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("B", C.c_int32), ("N", C.c_int32), ("H_q", C.c_int32),
                ("H_kv", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32), ("L_stride", C.c_int32),
                ("scale", C.c_float), ("parent_per_seq", C.c_int32), ("root_row", C.c_int32)]


class AttnBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("q", C.c_void_p), ("k_prefix", C.c_void_p),
                ("v_prefix", C.c_void_p), ("prefix_len", C.c_void_p), ("k_tree", C.c_void_p),
                ("v_tree", C.c_void_p), ("parent", C.c_void_p), ("out", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


class VerifyDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("B", C.c_int32), ("N", C.c_int32), ("V", C.c_int32),
                ("P", C.c_int32), ("variant", C.c_int32), ("gamma_max", C.c_int32),
                ("near_tie_eps", C.c_float), ("parent_per_seq", C.c_int32)]


class VerifyBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in (
        "target_logits", "draft_logits", "q_row", "parent", "cand_tok", "u_accept", "u_endpoint",
        "temperature", "n_accepted", "accepted_path", "out_tokens", "acc_child", "endpoint", "ratio",
        "flags", "residual_out", "workspace")] + [("workspace_bytes", C.c_size_t)]


class PagedKV(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("page_size", C.c_int32), ("n_pages", C.c_int32),
                ("max_pages_per_seq", C.c_int32), ("block_table", C.c_void_p)]


class DraftDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("B", C.c_int32), ("N", C.c_int32), ("V", C.c_int32),
                ("P", C.c_int32), ("variant", C.c_int32), ("near_tie_eps", C.c_float),
                ("parent_per_seq", C.c_int32)]


class DraftBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in (
        "draft_logits", "q_row", "parent", "u_draw", "temperature", "cand_tok", "flags")]


class CommitDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("B", C.c_int32), ("N", C.c_int32), ("H_kv", C.c_int32),
                ("d", C.c_int32), ("dtype", C.c_int32), ("L_stride", C.c_int32), ("gamma_max", C.c_int32),
                ("n_layers", C.c_int32), ("root_row", C.c_int32)]


class CommitBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in (
        "k_prefix", "v_prefix", "k_tree", "v_tree", "n_accepted", "accepted_path", "out_tokens",
        "prefix_len", "next_root", "flags")]


class FourbitKV(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("page_size", C.c_int32), ("n_pages", C.c_int32),
                ("max_pages_per_seq", C.c_int32)] + [(n, C.c_void_p) for n in (
                    "block_table", "k_codes", "v_codes", "k_scales", "v_scales")]


class RowsDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("T", C.c_int32), ("H_kv", C.c_int32), ("d", C.c_int32),
                ("dtype", C.c_int32), ("n_layers", C.c_int32), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
                ("k_layer_stride", C.c_int64), ("v_layer_stride", C.c_int64)]


class RowsBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("k", C.c_void_p), ("v", C.c_void_p), ("slot_map", C.c_void_p)]


class PageDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("B", C.c_int32), ("page_size", C.c_int32), ("n_pages", C.c_int32),
                ("max_pages_per_seq", C.c_int32), ("max_slots", C.c_int32)]


class PageBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in (
        "prefix_len", "want_len", "n_held", "block_table", "free_pages", "n_free", "slot_start", "slot_map", "flags")]


class LogitsDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in (
        "B", "N", "V", "R", "dtype", "parent_per_seq", "row_begin", "row_end", "hist_stride", "n_bias")]


class LogitsBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in (
        "logits", "out", "row_map", "parent", "cand_tok", "history", "hist_len", "prompt_len", "repetition",
        "presence", "frequency", "bias_tok", "bias_val", "mask")]


class StoreBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in ("k", "v", "slot_map", "k_pool", "v_pool")]


class ChunkDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in ("B", "T", "H_q", "H_kv", "d", "dtype", "L_stride")] + [
        ("scale", C.c_float), ("q_stride", C.c_int64)]


class ChunkBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in (
        "q", "k_pool", "v_pool", "chunk_start", "prefix_len", "out", "lse", "workspace")] + [("workspace_bytes", C.c_size_t)]


class SumsBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("last_rows", C.c_int32)] + [(n, C.c_void_p) for n in (
        "q", "k_pool", "chunk_start", "prefix_len", "lse", "sums")]


class EvictDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in (
        "B", "H_kv", "d", "dtype", "L_stride", "n_layers", "n_first", "n_recent")]


class EvictBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in (
        "k_pool", "v_pool", "sums", "prefix_len", "keep_len", "out_table", "kept", "flags")]


class LogprobDesc(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_int32) for n in ("rows", "R", "V", "dtype", "n_top")] + [("row_stride", C.c_int64)]


class LogprobBufs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32)] + [(n, C.c_void_p) for n in (
        "logits", "row_map", "tokens", "temperature", "logprob", "entropy", "rank", "top_tok", "top_logprob", "flags", "workspace")] + [
        ("workspace_bytes", C.c_size_t)]


_lib: Optional[C.CDLL] = None


def lib() -> C.CDLL:
    """Loads the in-tree library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2401_06706_amd.build` "
                "(there is no CPU fallback)")
        L = C.CDLL(LIB_PATH)
        L.mcsd_last_error.restype = C.c_char_p
        L.mcsd_version.restype = C.c_char_p
        L.mcsd_tree_validate.argtypes = [C.c_void_p, C.c_int32]
        L.mcsd_tree_validate.restype = C.c_int32
        L.mcsd_attn_workspace_bytes.argtypes = [C.POINTER(AttnDesc)]
        L.mcsd_attn_workspace_bytes.restype = C.c_size_t
        L.mcsd_verify_workspace_bytes.argtypes = [C.POINTER(VerifyDesc)]
        L.mcsd_verify_workspace_bytes.restype = C.c_size_t
        L.mcsd_tree_attn.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBufs), C.c_void_p]
        L.mcsd_tree_attn.restype = C.c_int32
        L.mcsd_tree_attn_static.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBufs), C.c_void_p]
        L.mcsd_tree_attn_static.restype = C.c_int32
        L.mcsd_attn_plan_override.argtypes = [C.c_int32, C.c_int32, C.c_int32]
        L.mcsd_attn_plan_override.restype = C.c_int32
        L.mcsd_tree_attn_paged.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBufs), C.POINTER(PagedKV), C.c_void_p]
        L.mcsd_tree_attn_paged.restype = C.c_int32
        L.mcsd_verify_sample.argtypes = [C.POINTER(VerifyDesc), C.POINTER(VerifyBufs), C.c_void_p]
        L.mcsd_verify_sample.restype = C.c_int32
        L.mcsd_verify_step.argtypes = [C.POINTER(AttnDesc), C.POINTER(AttnBufs), C.POINTER(VerifyDesc),
                                       C.POINTER(VerifyBufs), C.c_void_p]
        L.mcsd_verify_step.restype = C.c_int32
        L.mcsd_draft_sample.argtypes = [C.POINTER(DraftDesc), C.POINTER(DraftBufs), C.c_void_p]
        L.mcsd_draft_sample.restype = C.c_int32
        L.mcsd_tree_size.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.mcsd_tree_size.restype = C.c_int32
        L.mcsd_tree_build.argtypes = [C.c_void_p, C.c_int32, C.c_int32] + [C.c_void_p] * 5 + [C.c_int32, C.c_void_p]
        L.mcsd_tree_build.restype = C.c_int32
        L.mcsd_kv_commit.argtypes = [C.POINTER(CommitDesc), C.POINTER(CommitBufs), C.c_void_p]
        L.mcsd_kv_commit.restype = C.c_int32
        L.mcsd_kv_commit_paged.argtypes = [C.POINTER(CommitDesc), C.POINTER(CommitBufs), C.POINTER(PagedKV), C.c_void_p]
        L.mcsd_kv_commit_paged.restype = C.c_int32
        L.mcsd_attn_fourbit_workspace_bytes.argtypes = [C.POINTER(AttnDesc)]
        L.mcsd_attn_fourbit_workspace_bytes.restype = C.c_size_t
        for name, desc, bufs, kv in (("mcsd_tree_attn_fourbit", AttnDesc, AttnBufs, FourbitKV),
                                     ("mcsd_kv_commit_fourbit", CommitDesc, CommitBufs, FourbitKV),
                                     ("mcsd_kv_store_fourbit", RowsDesc, RowsBufs, FourbitKV),
                                     ("mcsd_kv_load_fourbit", RowsDesc, RowsBufs, FourbitKV),
                                     ("mcsd_kv_store_paged", RowsDesc, StoreBufs, PagedKV),
                                     ("mcsd_chunk_attn_paged", ChunkDesc, ChunkBufs, PagedKV),
                                     ("mcsd_attn_weight_sums", ChunkDesc, SumsBufs, PagedKV),
                                     ("mcsd_kv_evict_paged", EvictDesc, EvictBufs, PagedKV),
                                     ("mcsd_token_logprobs", LogprobDesc, LogprobBufs, None),
                                     ("mcsd_page_assign", PageDesc, PageBufs, None),
                                     ("mcsd_logits_rules", LogitsDesc, LogitsBufs, None)):
            f = getattr(L, name)
            f.argtypes = [C.POINTER(t) for t in (desc, bufs, kv) if t is not None] + [C.c_void_p]
            f.restype = C.c_int32
        for name, desc in (("mcsd_chunk_workspace_bytes", ChunkDesc), ("mcsd_logprob_workspace_bytes", LogprobDesc)):
            f = getattr(L, name)
            f.argtypes = [C.POINTER(desc)]
            f.restype = C.c_size_t
        L.mcsd_kernel_timing.argtypes = [C.c_int32]
        L.mcsd_kernel_timing.restype = C.c_int32
        L.mcsd_kernel_count.restype = C.c_int32
        L.mcsd_kernel_name.argtypes = [C.c_int32]
        L.mcsd_kernel_name.restype = C.c_char_p
        L.mcsd_kernel_timing_read.argtypes = [C.c_int32, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.mcsd_kernel_timing_read.restype = C.c_int32
        _lib = L
    return _lib


def _check(rc: int) -> None:
    if rc != 0:
        raise McsdError(rc, lib().mcsd_last_error().decode())


def _ptr(t: Optional[torch.Tensor], dtype=None, name: str = "tensor") -> Optional[int]:
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    return t.data_ptr()


# torch.cuda.current_stream().cuda_stream builds a Stream object for its handle: 2.7 us of a 6.7 us
# call, as much as the launch itself.  torch's own raw accessors give the handle in 0.2 us.
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is None or _current_device is None or not torch.cuda.is_initialized():
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(_current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def version() -> str:
    return lib().mcsd_version().decode()


def mcsd_tree_validate(parent_host) -> None:
    """parent_host: int32 numpy array / CPU tensor [N]."""
    import numpy as np
    a = np.ascontiguousarray(parent_host, dtype=np.int32)
    _check(lib().mcsd_tree_validate(a.ctypes.data_as(C.c_void_p), a.shape[0]))


# ------------------------------------------------------------------ tree attention
@dataclass
class AttnArgs:
    desc: AttnDesc
    bufs: AttnBufs
    keep: tuple       # tensors referenced by the raw pointers


def attn_desc(B, N, H_q, H_kv, d, dtype, L_stride, scale, parent_per_seq=False, root_row=False) -> AttnDesc:
    return AttnDesc(C.sizeof(AttnDesc), B, N, H_q, H_kv, d, dtype, L_stride, float(scale),
                    1 if parent_per_seq else 0, 1 if root_row else 0)


def mcsd_attn_workspace_bytes(desc: AttnDesc) -> int:
    n = lib().mcsd_attn_workspace_bytes(C.byref(desc))
    return int(n)


def attn_args(q, k_prefix, v_prefix, prefix_len, k_tree, v_tree, parent, out, scale,
              workspace: Optional[torch.Tensor] = None) -> AttnArgs:
    """Shapes: q/out [B][N][H_q][d]; k/v_prefix [B][H_kv][L_stride][d]; k/v_tree [B][H_kv][N][d];
    prefix_len int32 [B]; parent int32 [N] or [B][N].  If q, out, k_tree and v_tree have one row
    more than parent has entries, row 0 is the root (root_row = 1 in the descriptor)."""
    B, N, H_q, d = q.shape
    root_row = parent.shape[-1] == N - 1
    H_kv, L_stride = k_prefix.shape[1], k_prefix.shape[2]
    if q.dtype == torch.float32:
        dt = DTYPE_FP32
    elif q.dtype == torch.bfloat16:
        dt = DTYPE_BF16
    else:
        raise ValueError(f"unsupported dtype {q.dtype}")
    if tuple(k_prefix.shape) != (B, H_kv, L_stride, d) or tuple(v_prefix.shape) != (B, H_kv, L_stride, d):
        raise ValueError("k_prefix / v_prefix shape mismatch")
    if tuple(k_tree.shape) != (B, H_kv, N, d) or tuple(v_tree.shape) != (B, H_kv, N, d):
        raise ValueError("k_tree / v_tree shape mismatch")
    if tuple(out.shape) != (B, N, H_q, d) or tuple(prefix_len.shape) != (B,):
        raise ValueError("out / prefix_len shape mismatch")
    Np = N - 1 if root_row else N
    if tuple(parent.shape) not in ((Np,), (B, Np)):
        raise ValueError("parent must be [N] or [B][N]")
    desc = attn_desc(B, Np, H_q, H_kv, d, dt, L_stride, scale, parent.dim() == 2, root_row)
    bufs = AttnBufs(C.sizeof(AttnBufs), _ptr(q, q.dtype, "q"), _ptr(k_prefix, q.dtype, "k_prefix"),
                    _ptr(v_prefix, q.dtype, "v_prefix"), _ptr(prefix_len, torch.int32, "prefix_len"),
                    _ptr(k_tree, q.dtype, "k_tree"), _ptr(v_tree, q.dtype, "v_tree"),
                    _ptr(parent, torch.int32, "parent"), _ptr(out, q.dtype, "out"),
                    _ptr(workspace, None, "workspace"),
                    0 if workspace is None else workspace.numel() * workspace.element_size())
    return AttnArgs(desc, bufs, (q, k_prefix, v_prefix, prefix_len, k_tree, v_tree, parent, out, workspace))


def mcsd_tree_attn(args: AttnArgs, stream=None) -> None:
    _check(lib().mcsd_tree_attn(C.byref(args.desc), C.byref(args.bufs), _stream(stream)))


STATIC_SCRATCH_BYTES = 96 << 20


def mcsd_tree_attn_static(args: AttnArgs, stream=None) -> None:
    """mcsd_tree_attn without a workspace: the library's own static device buffer holds the partials."""
    _check(lib().mcsd_tree_attn_static(C.byref(args.desc), C.byref(args.bufs), _stream(stream)))


def mcsd_attn_plan_override(variant: int = 0, chunk_tiles: int = 0, target_items: int = 0) -> None:
    """Test / tuning aid: force the attention kernel variant (1..3), the segment length in 32-key
    tiles, or the item target of the launch plan, for all later calls (0 = automatic)."""
    _check(lib().mcsd_attn_plan_override(int(variant), int(chunk_tiles), int(target_items)))


def paged_attn_args(q, k_pool, v_pool, block_table, prefix_len, k_tree, v_tree, parent, out, scale, L_stride: int,
                    workspace: Optional[torch.Tensor] = None):
    """Like attn_args, with the prefix in pools [n_pages][H_kv][page_size][d] and block_table
    int32 [B][max_pages_per_seq].  Returns (AttnArgs, PagedKV)."""
    B, N, H_q, d = q.shape
    n_pages, H_kv, page_size, _ = k_pool.shape
    if tuple(v_pool.shape) != tuple(k_pool.shape) or k_pool.shape[3] != d:
        raise ValueError("pool shape mismatch")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B][max_pages_per_seq]")
    if q.dtype == torch.float32:
        dt = DTYPE_FP32
    elif q.dtype == torch.bfloat16:
        dt = DTYPE_BF16
    else:
        raise ValueError(f"unsupported dtype {q.dtype}")
    desc = attn_desc(B, N, H_q, H_kv, d, dt, L_stride, scale, parent.dim() == 2)
    bufs = AttnBufs(C.sizeof(AttnBufs), _ptr(q, q.dtype, "q"), _ptr(k_pool, q.dtype, "k_pool"),
                    _ptr(v_pool, q.dtype, "v_pool"), _ptr(prefix_len, torch.int32, "prefix_len"),
                    _ptr(k_tree, q.dtype, "k_tree"), _ptr(v_tree, q.dtype, "v_tree"),
                    _ptr(parent, torch.int32, "parent"), _ptr(out, q.dtype, "out"),
                    _ptr(workspace, None, "workspace"),
                    0 if workspace is None else workspace.numel() * workspace.element_size())
    paged = PagedKV(C.sizeof(PagedKV), page_size, n_pages, block_table.shape[1],
                    _ptr(block_table, torch.int32, "block_table"))
    keep = (q, k_pool, v_pool, block_table, prefix_len, k_tree, v_tree, parent, out, workspace)
    return AttnArgs(desc, bufs, keep), paged


def mcsd_tree_attn_paged(args: AttnArgs, paged: PagedKV, stream=None) -> None:
    _check(lib().mcsd_tree_attn_paged(C.byref(args.desc), C.byref(args.bufs), C.byref(paged), _stream(stream)))


# -------------------------------------------------------------------- verification
@dataclass
class VerifyArgs:
    desc: VerifyDesc
    bufs: VerifyBufs
    keep: tuple


def verify_args(target_logits, draft_logits, q_row, parent, cand_tok, u_accept, u_endpoint, temperature,
                n_accepted, accepted_path, out_tokens, acc_child, endpoint, flags, variant: int,
                ratio=None, residual_out=None, near_tie_eps: float = 1e-6) -> VerifyArgs:
    """Shapes: target_logits [B][1+N][V]; draft_logits [B][P][V]; q_row int32 [1+N] and parent int32 [N]
    (one tree for the batch) or q_row [B][1+N] and parent [B][N] (one tree per sequence);
    cand_tok int32 [B][N]; u_accept [B][N]; u_endpoint [B][1+N]; temperature [B];
    outputs n_accepted [B], accepted_path [B][gamma_max], out_tokens [B][gamma_max+1],
    acc_child / endpoint / flags [B][1+N], ratio [B][N] (optional), residual_out [B][1+N][V] (optional)."""
    B, rows, V = target_logits.shape
    N = rows - 1
    P = draft_logits.shape[1]
    gamma_max = accepted_path.shape[1]
    f32, i32 = torch.float32, torch.int32
    per_seq = parent.dim() == 2
    shapes = [(draft_logits, (B, P, V)), (q_row, (B, 1 + N) if per_seq else (1 + N,)),
              (parent, (B, N) if per_seq else (N,)), (cand_tok, (B, N)),
              (u_accept, (B, N)), (u_endpoint, (B, 1 + N)), (temperature, (B,)), (n_accepted, (B,)),
              (accepted_path, (B, gamma_max)), (out_tokens, (B, gamma_max + 1)), (acc_child, (B, 1 + N)),
              (endpoint, (B, 1 + N)), (flags, (B, 1 + N))]
    if ratio is not None:
        shapes.append((ratio, (B, N)))
    if residual_out is not None:
        shapes.append((residual_out, (B, 1 + N, V)))
    for t, shp in shapes:
        if tuple(t.shape) != shp:
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {shp}")
    desc = VerifyDesc(C.sizeof(VerifyDesc), B, N, V, P, int(variant), gamma_max, float(near_tie_eps),
                      1 if per_seq else 0)
    bufs = VerifyBufs(C.sizeof(VerifyBufs),
                      _ptr(target_logits, f32, "target_logits"), _ptr(draft_logits, f32, "draft_logits"),
                      _ptr(q_row, i32, "q_row"), _ptr(parent, i32, "parent"), _ptr(cand_tok, i32, "cand_tok"),
                      _ptr(u_accept, f32, "u_accept"), _ptr(u_endpoint, f32, "u_endpoint"),
                      _ptr(temperature, f32, "temperature"), _ptr(n_accepted, i32, "n_accepted"),
                      _ptr(accepted_path, i32, "accepted_path"), _ptr(out_tokens, i32, "out_tokens"),
                      _ptr(acc_child, i32, "acc_child"), _ptr(endpoint, i32, "endpoint"),
                      _ptr(ratio, f32, "ratio"), _ptr(flags, i32, "flags"),
                      _ptr(residual_out, f32, "residual_out"), None, 0)
    return VerifyArgs(desc, bufs, (target_logits, draft_logits, q_row, parent, cand_tok, u_accept,
                                   u_endpoint, temperature, n_accepted, accepted_path, out_tokens,
                                   acc_child, endpoint, ratio, flags, residual_out))


def mcsd_verify_workspace_bytes(desc: VerifyDesc) -> int:
    return int(lib().mcsd_verify_workspace_bytes(C.byref(desc)))


def mcsd_verify_sample(args: VerifyArgs, stream=None) -> None:
    _check(lib().mcsd_verify_sample(C.byref(args.desc), C.byref(args.bufs), _stream(stream)))


def mcsd_verify_step(attn: AttnArgs, verify: VerifyArgs, stream=None) -> None:
    _check(lib().mcsd_verify_step(C.byref(attn.desc), C.byref(attn.bufs), C.byref(verify.desc),
                                  C.byref(verify.bufs), _stream(stream)))


# ----------------------------------------------------------- draft-side candidates
@dataclass
class DraftArgs:
    desc: DraftDesc
    bufs: DraftBufs
    keep: tuple


def draft_args(draft_logits, q_row, parent, u_draw, temperature, cand_tok, flags, variant: int,
               near_tie_eps: float = 1e-6) -> DraftArgs:
    """Shapes: draft_logits [B][P][V]; q_row int32 [1+N] and parent int32 [N], or q_row [B][1+N] and
    parent [B][N] (one tree per sequence); u_draw [B][N]; temperature [B]; outputs cand_tok int32
    [B][N], flags int32 [B][N]."""
    B, P, V = draft_logits.shape
    per_seq = parent.dim() == 2
    N = parent.shape[-1]
    f32, i32 = torch.float32, torch.int32
    for t, shp in [(q_row, (B, 1 + N) if per_seq else (1 + N,)), (parent, (B, N) if per_seq else (N,)), (u_draw, (B, N)), (temperature, (B,)), (cand_tok, (B, N)), (flags, (B, N))]:
        if tuple(t.shape) != shp:
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {shp}")
    desc = DraftDesc(C.sizeof(DraftDesc), B, N, V, P, int(variant), float(near_tie_eps), 1 if per_seq else 0)
    bufs = DraftBufs(C.sizeof(DraftBufs), _ptr(draft_logits, f32, "draft_logits"), _ptr(q_row, i32, "q_row"),
                     _ptr(parent, i32, "parent"), _ptr(u_draw, f32, "u_draw"),
                     _ptr(temperature, f32, "temperature"), _ptr(cand_tok, i32, "cand_tok"),
                     _ptr(flags, i32, "flags"))
    return DraftArgs(desc, bufs, (draft_logits, q_row, parent, u_draw, temperature, cand_tok, flags))


def mcsd_draft_sample(args: DraftArgs, stream=None) -> None:
    _check(lib().mcsd_draft_sample(C.byref(args.desc), C.byref(args.bufs), _stream(stream)))


# ---------------------------------------------------- candidate tree and KV commit
def mcsd_tree_size(kconfig) -> tuple:
    """(N, P) of the k-ary candidate tree; host only."""
    import numpy as np
    kc = np.ascontiguousarray(kconfig, dtype=np.int32)
    n, pr = C.c_int32(0), C.c_int32(0)
    _check(lib().mcsd_tree_size(kc.ctypes.data_as(C.c_void_p), kc.shape[0], C.byref(n), C.byref(pr)))
    return int(n.value), int(pr.value)


def mcsd_tree_build(kconfig, parent, depth, q_row, prefix_len=None, position_ids=None, stream=None) -> None:
    """kconfig: host sequence; parent/depth int32 [N], q_row int32 [1+N] device tensors;
    position_ids int32 [B][N], or [B][1+N] with the root as entry 0 (optional, needs prefix_len int32 [B])."""
    import numpy as np
    kc = np.ascontiguousarray(kconfig, dtype=np.int32)
    N, _ = mcsd_tree_size(kc)
    i32 = torch.int32
    if tuple(parent.shape) != (N,) or tuple(depth.shape) != (N,) or tuple(q_row.shape) != (N + 1,):
        raise ValueError("parent / depth must be [N], q_row [1+N]")
    B = 1
    root_row = 0
    if position_ids is not None:
        B = position_ids.shape[0]
        root_row = 1 if position_ids.shape[1] == N + 1 else 0
        if tuple(position_ids.shape) != (B, N + root_row) or prefix_len is None or tuple(prefix_len.shape) != (B,):
            raise ValueError("position_ids must be [B][N] (or [B][1+N] with a root row) with prefix_len [B]")
    _check(lib().mcsd_tree_build(kc.ctypes.data_as(C.c_void_p), kc.shape[0], B, _ptr(prefix_len, i32, "prefix_len"),
                                 _ptr(parent, i32, "parent"), _ptr(depth, i32, "depth"), _ptr(q_row, i32, "q_row"),
                                 _ptr(position_ids, i32, "position_ids"), root_row, _stream(stream)))


@dataclass
class CommitArgs:
    desc: CommitDesc
    bufs: CommitBufs
    keep: tuple


def commit_args(k_prefix, v_prefix, k_tree, v_tree, n_accepted, accepted_path, out_tokens, prefix_len,
                next_root, flags, root_row: bool = False) -> CommitArgs:
    """k/v_prefix [n_layers][B][H_kv][L_stride][d] (or 4-D for one layer), k/v_tree [...][N][d]
    ([...][1+N][d] with root_row: row 0 = the root); n_accepted [B], accepted_path [B][gamma_max],
    out_tokens [B][gamma_max+1], prefix_len [B] (in/out), next_root [B], flags [B]."""
    if k_prefix.dim() == 4:
        n_layers, (B, H_kv, L_stride, d) = 1, k_prefix.shape
    else:
        n_layers, B, H_kv, L_stride, d = k_prefix.shape
    N = k_tree.shape[-2] - (1 if root_row else 0)
    lead = () if k_prefix.dim() == 4 else (n_layers,)
    if tuple(v_prefix.shape) != tuple(k_prefix.shape) or tuple(k_tree.shape) != lead + (B, H_kv, N + (1 if root_row else 0), d) or \
            tuple(v_tree.shape) != tuple(k_tree.shape):
        raise ValueError("cache shape mismatch")
    gamma_max = accepted_path.shape[1]
    for t, shp in [(n_accepted, (B,)), (accepted_path, (B, gamma_max)), (out_tokens, (B, gamma_max + 1)),
                   (prefix_len, (B,)), (next_root, (B,)), (flags, (B,))]:
        if tuple(t.shape) != shp:
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {shp}")
    if k_prefix.dtype == torch.float32:
        dt = DTYPE_FP32
    elif k_prefix.dtype == torch.bfloat16:
        dt = DTYPE_BF16
    else:
        raise ValueError(f"unsupported dtype {k_prefix.dtype}")
    i32 = torch.int32
    desc = CommitDesc(C.sizeof(CommitDesc), B, N, H_kv, d, dt, L_stride, gamma_max, n_layers, 1 if root_row else 0)
    bufs = CommitBufs(C.sizeof(CommitBufs), _ptr(k_prefix, k_prefix.dtype, "k_prefix"),
                      _ptr(v_prefix, k_prefix.dtype, "v_prefix"), _ptr(k_tree, k_prefix.dtype, "k_tree"),
                      _ptr(v_tree, k_prefix.dtype, "v_tree"), _ptr(n_accepted, i32, "n_accepted"),
                      _ptr(accepted_path, i32, "accepted_path"), _ptr(out_tokens, i32, "out_tokens"),
                      _ptr(prefix_len, i32, "prefix_len"), _ptr(next_root, i32, "next_root"),
                      _ptr(flags, i32, "flags"))
    return CommitArgs(desc, bufs, (k_prefix, v_prefix, k_tree, v_tree, n_accepted, accepted_path, out_tokens,
                                   prefix_len, next_root, flags))


def mcsd_kv_commit(args: CommitArgs, stream=None) -> None:
    _check(lib().mcsd_kv_commit(C.byref(args.desc), C.byref(args.bufs), _stream(stream)))


def paged_commit_args(k_pool, v_pool, block_table, k_tree, v_tree, n_accepted, accepted_path, out_tokens, prefix_len,
                      next_root, flags, L_stride: int, root_row: bool = False):
    """Like commit_args with the destination in pools [n_layers][n_pages][H_kv][page_size][d] (or 4-D
    for one layer) and block_table int32 [B][max_pages_per_seq].  Returns (CommitArgs, PagedKV)."""
    if k_pool.dim() == 4:
        n_layers, (n_pages, H_kv, page_size, d) = 1, k_pool.shape
    else:
        n_layers, n_pages, H_kv, page_size, d = k_pool.shape
    B, N = k_tree.shape[-4], k_tree.shape[-2] - (1 if root_row else 0)
    gamma_max = accepted_path.shape[1]
    if k_pool.dtype == torch.float32:
        dt = DTYPE_FP32
    elif k_pool.dtype == torch.bfloat16:
        dt = DTYPE_BF16
    else:
        raise ValueError(f"unsupported dtype {k_pool.dtype}")
    if tuple(v_pool.shape) != tuple(k_pool.shape) or tuple(v_tree.shape) != tuple(k_tree.shape):
        raise ValueError("pool / tree shape mismatch")
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError("block_table must be [B][max_pages_per_seq]")
    i32 = torch.int32
    desc = CommitDesc(C.sizeof(CommitDesc), B, N, H_kv, d, dt, L_stride, gamma_max, n_layers, 1 if root_row else 0)
    bufs = CommitBufs(C.sizeof(CommitBufs), _ptr(k_pool, k_pool.dtype, "k_pool"), _ptr(v_pool, k_pool.dtype, "v_pool"),
                      _ptr(k_tree, k_pool.dtype, "k_tree"), _ptr(v_tree, k_pool.dtype, "v_tree"),
                      _ptr(n_accepted, i32, "n_accepted"), _ptr(accepted_path, i32, "accepted_path"),
                      _ptr(out_tokens, i32, "out_tokens"), _ptr(prefix_len, i32, "prefix_len"),
                      _ptr(next_root, i32, "next_root"), _ptr(flags, i32, "flags"))
    paged = PagedKV(C.sizeof(PagedKV), page_size, n_pages, block_table.shape[1], _ptr(block_table, i32, "block_table"))
    keep = (k_pool, v_pool, block_table, k_tree, v_tree, n_accepted, accepted_path, out_tokens, prefix_len, next_root, flags)
    return CommitArgs(desc, bufs, keep), paged


def mcsd_kv_commit_paged(args: CommitArgs, paged: PagedKV, stream=None) -> None:
    _check(lib().mcsd_kv_commit_paged(C.byref(args.desc), C.byref(args.bufs), C.byref(paged), _stream(stream)))


# ------------------------------------------------------------ prefix cache in 4 bits
def _dtype_of(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return DTYPE_FP32
    if t.dtype == torch.bfloat16:
        return DTYPE_BF16
    raise ValueError(f"unsupported dtype {t.dtype}")


def _one_device(*tensors) -> int:
    """Index of the device that all these tensors lie on."""
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1 or next(iter(devices)).type != "cuda":
        raise ValueError(f"the tensors of a call must be on one GPU, got {sorted(str(d) for d in devices)}")
    return next(iter(devices)).index


def _launch(f, device: int, stream, *structs) -> None:
    """Calls f, whose tensors lie on `device`; the library enqueues on the current one."""
    current = _current_device() if _current_device is not None else torch.cuda.current_device()
    if current != device:
        raise ValueError(f"the tensors are on cuda:{device}, the current device is cuda:{current}")
    _check(f(*[C.byref(s) for s in structs], _stream(stream)))


def fourbit_shapes(n_pages: int, H_kv: int, page_size: int, d: int, n_layers: Optional[int] = None) -> tuple:
    """Shapes of the uint8 tensors of codes and of scales that hold n_pages pages (of n_layers layers) in 4 bits."""
    scales = (() if n_layers is None else (n_layers,)) + (n_pages, H_kv, page_size // 16, d // 32, 16)
    return scales + (16,), scales


@dataclass
class FourbitCache:
    kv: FourbitKV
    n_layers: int
    H_kv: int
    d: int
    layered: bool     # the pools have a leading axis of layers
    device: int
    keep: tuple


def fourbit_kv(k_codes, k_scales, v_codes, v_scales, block_table=None) -> FourbitCache:
    """A paged prefix cache held in 4 bits: uint8 tensors of the shapes of fourbit_shapes (pages in units of 16 rows; a leading axis of
    layers where they hold several) and block_table int32 [B][max_pages_per_seq] (not needed by rows in and out)."""
    if k_codes.dim() not in (6, 7) or tuple(k_codes.shape[-2:]) != (16, 16):
        raise ValueError("codes must be [n_pages][H_kv][page_size/16][d/32][16][16], with or without layers in front")
    for t, shp in [(v_codes, k_codes.shape), (k_scales, k_codes.shape[:-1]), (v_scales, k_codes.shape[:-1])]:
        if tuple(t.shape) != tuple(shp):
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {tuple(shp)}")
    if block_table is not None and block_table.dim() != 2:
        raise ValueError("block_table must be [B][max_pages_per_seq]")
    layered = k_codes.dim() == 7
    n_pages, H_kv, tiles, blocks = k_codes.shape[-6:-2]
    u8 = torch.uint8
    kv = FourbitKV(C.sizeof(FourbitKV), 16 * tiles, n_pages, 1 if block_table is None else block_table.shape[1],
                   _ptr(block_table, torch.int32, "block_table"), _ptr(k_codes, u8, "k_codes"), _ptr(v_codes, u8, "v_codes"),
                   _ptr(k_scales, u8, "k_scales"), _ptr(v_scales, u8, "v_scales"))
    device = _one_device(k_codes, k_scales, v_codes, v_scales, block_table)
    return FourbitCache(kv, k_codes.shape[0] if layered else 1, H_kv, 32 * blocks, layered, device,
                        (k_codes, k_scales, v_codes, v_scales, block_table))


@dataclass
class FourbitAttnArgs:
    desc: AttnDesc
    bufs: AttnBufs
    kv: FourbitKV
    device: int
    keep: tuple


def mcsd_attn_fourbit_workspace_bytes(desc: AttnDesc) -> int:
    return int(lib().mcsd_attn_fourbit_workspace_bytes(C.byref(desc)))


def fourbit_attn_args(q, cache: FourbitCache, prefix_len, k_tree, v_tree, parent, out, scale, L_stride: int,
                      workspace: Optional[torch.Tensor] = None) -> FourbitAttnArgs:
    """Like paged_attn_args with the prefix in a FourbitCache (one layer, with a block table).  If q, out, k_tree and
    v_tree have one row more than parent has entries, row 0 is the root."""
    B, rows, H_q, d = q.shape
    root_row = parent.shape[-1] == rows - 1
    N = rows - 1 if root_row else rows
    H_kv = cache.H_kv
    if cache.n_layers != 1 or cache.d != d:
        raise ValueError("the cache must hold one layer of the query's head dimension")
    if cache.keep[4] is None or cache.keep[4].shape[0] != B:
        raise ValueError("block_table must be [B][max_pages_per_seq]")
    for t, shp in [(k_tree, (B, H_kv, rows, d)), (v_tree, (B, H_kv, rows, d)), (out, (B, rows, H_q, d)), (prefix_len, (B,))]:
        if tuple(t.shape) != shp:
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {shp}")
    if tuple(parent.shape) not in ((N,), (B, N)):
        raise ValueError("parent must be [N] or [B][N]")
    desc = attn_desc(B, N, H_q, H_kv, d, _dtype_of(q), L_stride, scale, parent.dim() == 2, root_row)
    bufs = AttnBufs(C.sizeof(AttnBufs), _ptr(q, q.dtype, "q"), None, None, _ptr(prefix_len, torch.int32, "prefix_len"),
                    _ptr(k_tree, q.dtype, "k_tree"), _ptr(v_tree, q.dtype, "v_tree"), _ptr(parent, torch.int32, "parent"),
                    _ptr(out, q.dtype, "out"), _ptr(workspace, None, "workspace"),
                    0 if workspace is None else workspace.numel() * workspace.element_size())
    device = _one_device(q, cache.keep[0], prefix_len, k_tree, v_tree, parent, out, workspace)
    return FourbitAttnArgs(desc, bufs, cache.kv, device, (q, cache, prefix_len, k_tree, v_tree, parent, out, workspace))


def mcsd_tree_attn_fourbit(args: FourbitAttnArgs, stream=None) -> None:
    _launch(lib().mcsd_tree_attn_fourbit, args.device, stream, args.desc, args.bufs, args.kv)


@dataclass
class FourbitCommitArgs:
    desc: CommitDesc
    bufs: CommitBufs
    kv: FourbitKV
    device: int
    keep: tuple


def fourbit_commit_args(cache: FourbitCache, k_tree, v_tree, n_accepted, accepted_path, out_tokens, prefix_len,
                        next_root, flags, L_stride: int, root_row: bool = False) -> FourbitCommitArgs:
    """Like paged_commit_args with the destination a FourbitCache (with a block table); k/v_tree fp32 or bf16."""
    lead = (cache.n_layers,) if cache.layered else ()
    B, N = k_tree.shape[-4], k_tree.shape[-2] - (1 if root_row else 0)
    gamma_max = accepted_path.shape[1]
    tree_shape = lead + (B, cache.H_kv, N + (1 if root_row else 0), cache.d)
    if cache.keep[4] is None or cache.keep[4].shape[0] != B:
        raise ValueError("block_table must be [B][max_pages_per_seq]")
    for t, shp in [(k_tree, tree_shape), (v_tree, tree_shape), (n_accepted, (B,)), (accepted_path, (B, gamma_max)),
                   (out_tokens, (B, gamma_max + 1)), (prefix_len, (B,)), (next_root, (B,)), (flags, (B,))]:
        if tuple(t.shape) != shp:
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {shp}")
    i32 = torch.int32
    desc = CommitDesc(C.sizeof(CommitDesc), B, N, cache.H_kv, cache.d, _dtype_of(k_tree), L_stride, gamma_max, cache.n_layers,
                      1 if root_row else 0)
    bufs = CommitBufs(C.sizeof(CommitBufs), None, None, _ptr(k_tree, k_tree.dtype, "k_tree"), _ptr(v_tree, k_tree.dtype, "v_tree"),
                      _ptr(n_accepted, i32, "n_accepted"), _ptr(accepted_path, i32, "accepted_path"),
                      _ptr(out_tokens, i32, "out_tokens"), _ptr(prefix_len, i32, "prefix_len"),
                      _ptr(next_root, i32, "next_root"), _ptr(flags, i32, "flags"))
    keep = (cache, k_tree, v_tree, n_accepted, accepted_path, out_tokens, prefix_len, next_root, flags)
    return FourbitCommitArgs(desc, bufs, cache.kv, _one_device(cache.keep[0], *keep[1:]), keep)


def mcsd_kv_commit_fourbit(args: FourbitCommitArgs, stream=None) -> None:
    _launch(lib().mcsd_kv_commit_fourbit, args.device, stream, args.desc, args.bufs, args.kv)


@dataclass
class RowsArgs:
    desc: RowsDesc
    bufs: RowsBufs
    kv: FourbitKV
    device: int
    keep: tuple


def _rows_ptr(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    H_kv, d = t.shape[-2:]
    if t.numel() and (t.stride(-1) != 1 or (H_kv > 1 and t.stride(-2) != d)):
        raise ValueError(f"{name}: a token's row [H_kv][d] must be contiguous")
    return t.data_ptr()


def fourbit_rows_args(k, v, slot_map, cache: FourbitCache) -> RowsArgs:
    """Rows of tokens for a store into, or a load from, the cache: k, v [T][H_kv][d] ([n_layers][T][H_kv][d] where the
    cache has layers), a token's row contiguous, any stride from row to row; slot_map int32 [T]."""
    T = slot_map.shape[0]
    shape = ((cache.n_layers,) if cache.layered else ()) + (T, cache.H_kv, cache.d)
    if slot_map.dim() != 1 or tuple(k.shape) != shape or tuple(v.shape) != shape or k.dtype != v.dtype:
        raise ValueError(f"k and v must be {shape} of one dtype, slot_map [T]")
    row = cache.H_kv * cache.d
    stride = lambda t: t.stride(-3) if T > 1 else row
    layer = lambda t: t.stride(0) if cache.n_layers > 1 else 0
    desc = RowsDesc(C.sizeof(RowsDesc), T, cache.H_kv, cache.d, _dtype_of(k), cache.n_layers, stride(k), stride(v), layer(k), layer(v))
    bufs = RowsBufs(C.sizeof(RowsBufs), _rows_ptr(k, "k"), _rows_ptr(v, "v"), _ptr(slot_map, torch.int32, "slot_map"))
    return RowsArgs(desc, bufs, cache.kv, _one_device(k, v, slot_map, cache.keep[0]), (k, v, slot_map, cache))


def mcsd_kv_store_fourbit(args: RowsArgs, stream=None) -> None:
    _launch(lib().mcsd_kv_store_fourbit, args.device, stream, args.desc, args.bufs, args.kv)


def mcsd_kv_load_fourbit(args: RowsArgs, stream=None) -> None:
    _launch(lib().mcsd_kv_load_fourbit, args.device, stream, args.desc, args.bufs, args.kv)


# ------------------------------------------------- prompts in chunks over a paged cache
def _pools(k_pool, v_pool=None):
    """(n_layers, n_pages, H_kv, page_size, d) of pools [n_pages][H_kv][page_size][d], with or without layers in front."""
    if k_pool.dim() not in (4, 5) or (v_pool is not None and (tuple(v_pool.shape) != tuple(k_pool.shape) or v_pool.dtype != k_pool.dtype)):
        raise ValueError("pools must be [n_pages][H_kv][page_size][d], with or without layers in front, keys and values alike")
    return (1,) * (5 - k_pool.dim()) + tuple(k_pool.shape)


def _paged(k_pool, block_table=None) -> PagedKV:
    if block_table is not None and block_table.dim() != 2:
        raise ValueError("block_table must be [B][max_pages_per_seq]")
    return PagedKV(C.sizeof(PagedKV), k_pool.shape[-2], k_pool.shape[-4], 0 if block_table is None else block_table.shape[1],
                   _ptr(block_table, torch.int32, "block_table"))


def _bytes_of(workspace) -> int:
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


@dataclass
class StoreArgs:
    desc: RowsDesc
    bufs: StoreBufs
    paged: PagedKV
    device: int
    keep: tuple


def store_args(k, v, slot_map, k_pool, v_pool) -> StoreArgs:
    """Rows of tokens for a store into pools [n_pages][H_kv][page_size][d]: k, v [T][H_kv][d] (layers in front of both where the
    pools have them), a token's row contiguous, any stride from row to row; slot_map int32 [T]."""
    n_layers, _, H_kv, _, d = _pools(k_pool, v_pool)
    T = slot_map.shape[0]
    shape = tuple(k_pool.shape[:-4]) + (T, H_kv, d)
    if slot_map.dim() != 1 or tuple(k.shape) != shape or tuple(v.shape) != shape or k.dtype != k_pool.dtype or v.dtype != k_pool.dtype:
        raise ValueError(f"k and v must be {shape} of the pools' dtype, slot_map [T]")
    stride = lambda t: t.stride(-3) if T > 1 else H_kv * d
    layer = lambda t: t.stride(0) if n_layers > 1 else 0
    desc = RowsDesc(C.sizeof(RowsDesc), T, H_kv, d, _dtype_of(k), n_layers, stride(k), stride(v), layer(k), layer(v))
    bufs = StoreBufs(C.sizeof(StoreBufs), _rows_ptr(k, "k"), _rows_ptr(v, "v"), _ptr(slot_map, torch.int32, "slot_map"),
                     _ptr(k_pool, k.dtype, "k_pool"), _ptr(v_pool, k.dtype, "v_pool"))
    return StoreArgs(desc, bufs, _paged(k_pool), _one_device(k, v, slot_map, k_pool, v_pool), (k, v, slot_map, k_pool, v_pool))


def mcsd_kv_store_paged(args: StoreArgs, stream=None) -> None:
    _launch(lib().mcsd_kv_store_paged, args.device, stream, args.desc, args.bufs, args.paged)


def chunk_desc(q, k_pool, block_table, scale: float, L_stride: int) -> ChunkDesc:
    """q [T][H_q][d] (a row contiguous, any stride from row to row) over pools [n_pages][H_kv][page_size][d] (one layer)."""
    n_layers, _, H_kv, _, d = _pools(k_pool)
    if n_layers != 1 or k_pool.dim() != 4 or q.dim() != 3 or q.shape[2] != d or q.dtype != k_pool.dtype or block_table.dim() != 2:
        raise ValueError("q must be [T][H_q][d] of the pools' dtype and head dimension, the pools of one layer, block_table [B][max_pages_per_seq]")
    T, H_q, _ = q.shape
    return ChunkDesc(C.sizeof(ChunkDesc), block_table.shape[0], T, H_q, H_kv, d, _dtype_of(q), int(L_stride), float(scale),
                     q.stride(0) if T > 1 else H_q * d)


def mcsd_chunk_workspace_bytes(desc: ChunkDesc) -> int:
    return int(lib().mcsd_chunk_workspace_bytes(C.byref(desc)))


@dataclass
class ChunkArgs:
    desc: ChunkDesc
    bufs: C.Structure
    paged: PagedKV
    device: int
    keep: tuple


def _chunk_shapes(desc, *pairs) -> None:
    for t, shp in pairs:
        if t is not None and tuple(t.shape) != shp:
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {shp}")


def chunk_attn_args(q, k_pool, v_pool, block_table, chunk_start, prefix_len, out, scale, L_stride: int, lse=None,
                    workspace: Optional[torch.Tensor] = None) -> ChunkArgs:
    """q as for chunk_desc, out [T][H_q][d], lse fp32 [T][H_q] or None; block_table int32 [B][max_pages_per_seq], chunk_start int32
    [B+1], prefix_len int32 [B]."""
    desc = chunk_desc(q, k_pool, block_table, scale, L_stride)
    _pools(k_pool, v_pool)
    _chunk_shapes(desc, (out, tuple(q.shape)), (lse, tuple(q.shape[:2])), (chunk_start, (desc.B + 1,)), (prefix_len, (desc.B,)))
    bufs = ChunkBufs(C.sizeof(ChunkBufs), _rows_ptr(q, "q"), _ptr(k_pool, q.dtype, "k_pool"), _ptr(v_pool, q.dtype, "v_pool"),
                     _ptr(chunk_start, torch.int32, "chunk_start"), _ptr(prefix_len, torch.int32, "prefix_len"), _ptr(out, q.dtype, "out"),
                     _ptr(lse, torch.float32, "lse"), _ptr(workspace, None, "workspace"), _bytes_of(workspace))
    keep = (q, k_pool, v_pool, block_table, chunk_start, prefix_len, out, lse, workspace)
    return ChunkArgs(desc, bufs, _paged(k_pool, block_table), _one_device(*keep), keep)


def mcsd_chunk_attn_paged(args: ChunkArgs, stream=None) -> None:
    _launch(lib().mcsd_chunk_attn_paged, args.device, stream, args.desc, args.bufs, args.paged)


# ------------------------------------------------------ eviction by attention weight
def weight_sums_args(q, k_pool, block_table, chunk_start, prefix_len, lse, sums, scale, last_rows: int = 0) -> ChunkArgs:
    """As chunk_attn_args; lse fp32 [T][H_q] as written there, sums fp32 [B][H_kv][L_stride] (in/out)."""
    if sums.dim() != 3:
        raise ValueError("sums must be [B][H_kv][L_stride]")
    desc = chunk_desc(q, k_pool, block_table, scale, sums.shape[2])
    _chunk_shapes(desc, (sums, (desc.B, desc.H_kv, desc.L_stride)), (lse, tuple(q.shape[:2])), (chunk_start, (desc.B + 1,)), (prefix_len, (desc.B,)))
    bufs = SumsBufs(C.sizeof(SumsBufs), int(last_rows), _rows_ptr(q, "q"), _ptr(k_pool, q.dtype, "k_pool"), _ptr(chunk_start, torch.int32, "chunk_start"),
                    _ptr(prefix_len, torch.int32, "prefix_len"), _ptr(lse, torch.float32, "lse"), _ptr(sums, torch.float32, "sums"))
    keep = (q, k_pool, block_table, chunk_start, prefix_len, lse, sums)
    return ChunkArgs(desc, bufs, _paged(k_pool, block_table), _one_device(*keep), keep)


def mcsd_attn_weight_sums(args: ChunkArgs, stream=None) -> None:
    _launch(lib().mcsd_attn_weight_sums, args.device, stream, args.desc, args.bufs, args.paged)


@dataclass
class EvictArgs:
    desc: EvictDesc
    bufs: EvictBufs
    paged: PagedKV
    device: int
    keep: tuple


def evict_args(k_pool, v_pool, block_table, sums, prefix_len, keep_len, kept, flags, n_first: int, n_recent: int, out_table=None) -> EvictArgs:
    """Pools [n_layers][n_pages][H_kv][page_size][d] with sums fp32 and kept int32 [n_layers][B][H_kv][L_stride] (or all without
    layers); block_table and out_table int32 [B][max_pages_per_seq]; prefix_len, keep_len, flags int32 [B]."""
    n_layers, _, H_kv, _, d = _pools(k_pool, v_pool)
    if block_table.dim() != 2 or sums.dim() != k_pool.dim() - 1:
        raise ValueError("block_table must be [B][max_pages_per_seq], sums [B][H_kv][L_stride] with layers in front where the pools have them")
    B, L_stride = block_table.shape[0], sums.shape[-1]
    _chunk_shapes(None, (sums, tuple(k_pool.shape[:-4]) + (B, H_kv, L_stride)), (kept, tuple(sums.shape)), (out_table, tuple(block_table.shape)),
                  (prefix_len, (B,)), (keep_len, (B,)), (flags, (B,)))
    i32 = torch.int32
    desc = EvictDesc(C.sizeof(EvictDesc), B, H_kv, d, _dtype_of(k_pool), L_stride, n_layers, int(n_first), int(n_recent))
    bufs = EvictBufs(C.sizeof(EvictBufs), _ptr(k_pool, k_pool.dtype, "k_pool"), _ptr(v_pool, k_pool.dtype, "v_pool"), _ptr(sums, torch.float32, "sums"),
                     _ptr(prefix_len, i32, "prefix_len"), _ptr(keep_len, i32, "keep_len"), _ptr(out_table, i32, "out_table"),
                     _ptr(kept, i32, "kept"), _ptr(flags, i32, "flags"))
    keep = (k_pool, v_pool, block_table, sums, prefix_len, keep_len, kept, flags, out_table)
    return EvictArgs(desc, bufs, _paged(k_pool, block_table), _one_device(*keep), keep)


def mcsd_kv_evict_paged(args: EvictArgs, stream=None) -> None:
    _launch(lib().mcsd_kv_evict_paged, args.device, stream, args.desc, args.bufs, args.paged)


# --------------------------------------------------------- log probabilities of tokens
@dataclass
class LogprobArgs:
    desc: LogprobDesc
    bufs: LogprobBufs
    device: int
    keep: tuple


def logprob_desc(logits, tokens, n_top: int = 0) -> LogprobDesc:
    """logits [R][V] (a row contiguous, any stride from row to row), tokens [rows]."""
    R, V = logits.shape
    if V > 1 and logits.stride(1) != 1:
        raise ValueError("a row of logits must be contiguous")
    return LogprobDesc(C.sizeof(LogprobDesc), tokens.shape[0], R, V, _dtype_of(logits), int(n_top), logits.stride(0) if R > 1 else V)


def mcsd_logprob_workspace_bytes(desc: LogprobDesc) -> int:
    return int(lib().mcsd_logprob_workspace_bytes(C.byref(desc)))


def logprob_args(logits, tokens, logprob, entropy, rank, top_tok, top_logprob, flags, temperature=None, row_map=None,
                 workspace: Optional[torch.Tensor] = None) -> LogprobArgs:
    """logits fp32 or bf16 [R][V]; int32 tokens, flags, rank (or None), row_map (or None: row i) [rows]; fp32 logprob, entropy
    (or None), temperature (or None: 1) [rows]; top_tok int32 and top_logprob fp32 [rows][n_top] (or both None)."""
    if not logits.is_cuda:
        raise ValueError("logits must be a device tensor")
    if (top_tok is None) != (top_logprob is None):
        raise ValueError("top_tok and top_logprob come together")
    rows, n_top = tokens.shape[0], 0 if top_tok is None else top_tok.shape[1]
    _chunk_shapes(None, *[(t, (rows,)) for t in (tokens, logprob, entropy, rank, flags, temperature, row_map)], (top_tok, (rows, n_top)),
                  (top_logprob, (rows, n_top)))
    f32, i32 = torch.float32, torch.int32
    desc = logprob_desc(logits, tokens, n_top)
    keep = (row_map, tokens, temperature, logprob, entropy, rank, top_tok, top_logprob, flags)
    types = (i32, i32, f32, f32, f32, i32, i32, f32, i32)
    names = [n for n, _ in LogprobBufs._fields_[2:11]]
    bufs = LogprobBufs(C.sizeof(LogprobBufs), logits.data_ptr(), *[_ptr(t, ty, n) for t, ty, n in zip(keep, types, names)],
                       _ptr(workspace, None, "workspace"), _bytes_of(workspace))
    if n_top == 0:
        bufs.top_tok = bufs.top_logprob = None
    return LogprobArgs(desc, bufs, _one_device(logits, *keep, workspace), (logits, workspace) + keep)


def mcsd_token_logprobs(args: LogprobArgs, stream=None) -> None:
    _launch(lib().mcsd_token_logprobs, args.device, stream, args.desc, args.bufs)


# ------------------------------------------------------------------ pages from lengths
@dataclass
class PageArgs:
    desc: PageDesc
    bufs: PageBufs
    device: int
    keep: tuple


def page_args(prefix_len, want_len, n_held, block_table, free_pages, n_free, flags, page_size: int,
              slot_start=None, slot_map=None) -> PageArgs:
    """int32 tensors: prefix_len, want_len, n_held, flags [B]; block_table [B][max_pages_per_seq]; free_pages [n_pages];
    n_free [1]; slot_start [B+1] and slot_map [max_slots] (both or neither)."""
    B, width = block_table.shape
    if (slot_start is None) != (slot_map is None):
        raise ValueError("slot_start and slot_map come together")
    shapes = [(t, (B,)) for t in (prefix_len, want_len, n_held, flags)] + [(n_free, (1,))]
    if slot_map is not None:
        shapes += [(slot_start, (B + 1,))]
    for t, shp in shapes:
        if tuple(t.shape) != shp:
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {shp}")
    if free_pages.dim() != 1 or (slot_map is not None and slot_map.dim() != 1):
        raise ValueError("free_pages and slot_map must be vectors")
    i32 = torch.int32
    desc = PageDesc(C.sizeof(PageDesc), B, int(page_size), free_pages.shape[0], width, 0 if slot_map is None else slot_map.shape[0])
    keep = (prefix_len, want_len, n_held, block_table, free_pages, n_free, slot_start, slot_map, flags)
    names = ("prefix_len", "want_len", "n_held", "block_table", "free_pages", "n_free", "slot_start", "slot_map", "flags")
    bufs = PageBufs(C.sizeof(PageBufs), *[_ptr(t, i32, n) for t, n in zip(keep, names)])
    return PageArgs(desc, bufs, _one_device(*keep), keep)


def mcsd_page_assign(args: PageArgs, stream=None) -> None:
    _launch(lib().mcsd_page_assign, args.device, stream, args.desc, args.bufs)


# --------------------------------------------------------------------- rules on logits
@dataclass
class LogitsArgs:
    desc: LogitsDesc
    bufs: LogitsBufs
    device: int
    keep: tuple


def logits_args(logits, out, parent=None, cand_tok=None, history=None, hist_len=None, prompt_len=None, repetition=None,
                presence=None, frequency=None, bias_tok=None, bias_val=None, mask=None, row_map=None, rows=None) -> LogitsArgs:
    """logits [B][R][V] fp32 or bf16, out [B][R][V] fp32 (the logits themselves: in place); parent int32 [N] or [B][N], cand_tok int32
    [B][N] (neither: the root's row alone); history int32 [B][S] with hist_len, prompt_len int32 [B]; repetition, presence,
    frequency fp32 [B]; bias_tok int32 and bias_val fp32 [B][n]; mask int32 [B][R][ceil(V/32)] (32 tokens a word);
    row_map int32 [1+N] or [B][1+N] (as parent); rows: (begin, end) of the tree rows dealt with, all by default."""
    B, R, V = logits.shape
    N = 0 if parent is None else parent.shape[-1]
    per_seq = parent is not None and parent.dim() == 2
    if (parent is None) != (cand_tok is None) or (history is None) != (hist_len is None) or (bias_tok is None) != (bias_val is None):
        raise ValueError("parent and cand_tok, history and hist_len, bias_tok and bias_val come together")
    if row_map is not None and parent is None:
        per_seq = row_map.dim() == 2
    f32, i32 = torch.float32, torch.int32
    S = 0 if history is None else history.shape[1]
    n_bias = 0 if bias_tok is None else bias_tok.shape[1]
    shapes = [(out, (B, R, V)), (parent, (B, N) if per_seq else (N,)), (cand_tok, (B, N)), (history, (B, S)),
              (row_map, (B, 1 + N) if per_seq else (1 + N,)), (bias_tok, (B, n_bias)), (bias_val, (B, n_bias)), (mask, (B, R, (V + 31) // 32))]
    shapes += [(t, (B,)) for t in (hist_len, prompt_len, repetition, presence, frequency)]
    for t, shp in shapes:
        if t is not None and tuple(t.shape) != shp:
            raise ValueError(f"shape mismatch: got {tuple(t.shape)}, expected {shp}")
    begin, end = (0, 1 + N) if rows is None else rows
    desc = LogitsDesc(C.sizeof(LogitsDesc), B, N, V, R, _dtype_of(logits), 1 if per_seq else 0, int(begin), int(end), S, n_bias)
    keep = (logits, out, row_map, parent, cand_tok, history, hist_len, prompt_len, repetition, presence, frequency, bias_tok, bias_val, mask)
    types = (logits.dtype, f32, i32, i32, i32, i32, i32, i32, f32, f32, f32, i32, f32, i32)
    names = [n for n, _ in LogitsBufs._fields_[1:]]
    bufs = LogitsBufs(C.sizeof(LogitsBufs), *[None if t is None or t.numel() == 0 else _ptr(t, ty, n) for t, ty, n in zip(keep, types, names)])
    return LogitsArgs(desc, bufs, _one_device(*keep), keep)


def mcsd_logits_rules(args: LogitsArgs, stream=None) -> None:
    _launch(lib().mcsd_logits_rules, args.device, stream, args.desc, args.bufs)


# ------------------------------------------------------------------- profiling aid
def mcsd_kernel_timing(enable: bool) -> None:
    _check(lib().mcsd_kernel_timing(1 if enable else 0))


def mcsd_kernel_timing_read() -> dict:
    """{kernel name: (total ms, launches)} since timing was enabled; waits for the events."""
    out = {}
    L = lib()
    for i in range(L.mcsd_kernel_count()):
        ms, n = C.c_double(0.0), C.c_int64(0)
        _check(L.mcsd_kernel_timing_read(i, C.byref(ms), C.byref(n)))
        out[L.mcsd_kernel_name(i).decode()] = (ms.value, n.value)
    return out
