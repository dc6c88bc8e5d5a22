"""How the library lays out a launch of attention over the 4-bit cache, for tests that are meant to reach a certain kernel: its own plan
(read on the host, nothing touches a GPU), and how the sequences of a batch are then cut, after the rule in fourbit_attn.hip."""
import ctypes as C

import numpy as np

from paper_2401_06706_amd import binding as M

KT = 32


class Plan(C.Structure):
    _fields_ = [("rows_per_kv", C.c_int), ("n_row_tiles", C.c_int), ("row_tile", C.c_int), ("n_segments_max", C.c_int), ("n_segments", C.c_int),
                ("target", C.c_int), ("bias", C.c_float), ("min_seg", C.c_int), ("whole", C.c_int), ("ws_bytes", C.c_size_t)]


def plan_of(desc):
    f = getattr(M.lib(), "_ZN4mcsd17make_fourbit_planERK14mcsd_attn_descPNS_11FourbitPlanE")
    f.restype = C.c_bool
    p = Plan()
    assert f(C.byref(desc), C.byref(p))
    assert p.ws_bytes == M.mcsd_attn_fourbit_workspace_bytes(desc)
    return p


def form_of(desc, plan):
    """(padded head dimension, 16-row tiles per wavefront, row groups) of the kernel that the launch takes."""
    forms = {16: (1, 1), 32: (2, 1), 64: (2, 2), 128: (2, 4)}
    return (64 if desc.d <= 64 else 128 if desc.d <= 128 else 256,) + forms[plan.row_tile]


def segments_of(desc, plan, lens):
    """Segments of every sequence."""
    if plan.n_segments_max == 1:
        return [1] * len(lens)
    rows = desc.N + desc.root_row
    tiles = [-(-max(0, min(n, desc.L_stride)) // KT) + -(-rows // KT) for n in lens]
    units = desc.H_kv * plan.n_row_tiles
    chunk = max(plan.min_seg, int(np.ceil(np.float32(sum(tiles)) * np.float32(units / plan.target))))
    per_chunk = np.float32(1) / np.float32(chunk)
    return [1 if t <= plan.whole else max(1, min(plan.n_segments_max, int(np.float32(t) * per_chunk + np.float32(plan.bias)))) for t in tiles]
