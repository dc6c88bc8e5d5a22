"""Attention over the 4-bit cache at head dimensions other than 128: softmax weights reach PV to 2^-17, as in the framework's attention over caches of full
precision."""
import numpy as np
import pytest
import torch

from tests import fourbit_ref as F
from tests.fourbit_plan import form_of, plan_of, segments_of
from tests.test_gpu_fourbit import AttnCase, f64, random_tree

pytestmark = pytest.mark.gpu


def expected(q, k, v, k_tree, v_tree, vis, scale):
    """out [N][H_q][d] of one sequence in 64 bits, and how far off it may be.  With weights p_j (sum 1):
      a weight enters PV as two bf16 terms, at most 2^-17 of it off: sum p_j |v_j| 2^-17;
      a score: d products in fp32 and their scaling, at most (d + 2) 2^-24 sum |q k| scale + 4 2^-24 (|s| + |max|), which scales a weight by as
      much, here and in the sum that it is divided by (hence twice);
      sums of weights and of PV: at most 2^10 roundings of 2^-24 (up to 5000 keys in steps of 32, two terms, streams and segments joined): 2^-14 of
      sum p_j |v_j|;
      the output: half a step of bf16, 2^-8 of it (2^-134 where it is subnormal)."""
    N, H_q, d = q.shape
    G, L = H_q // k.shape[0], k.shape[1]
    out, bound = np.empty_like(q), np.empty_like(q)
    for h in range(H_q):
        kk, vv = np.concatenate((k[h // G], k_tree[h // G])), np.concatenate((v[h // G], v_tree[h // G]))
        s = q[:, h] @ kk.T * scale
        mag = np.abs(q[:, h]) @ np.abs(kk).T * scale
        s[:, L:][~vis] = -np.inf
        top = s.max(-1, keepdims=True)
        p = np.exp(s - top)
        p /= p.sum(-1, keepdims=True)
        ds = 2.0 ** -24 * ((d + 2) * mag + 4 * (np.where(np.isfinite(s), np.abs(s), 0) + np.abs(top)))
        out[:, h] = p @ vv
        bound[:, h] = (p * (2.0 ** -17 + 2.0 ** -14 + 2 * (ds + ds.max(-1, keepdims=True)))) @ np.abs(vv) + np.abs(out[:, h]) * 2.0 ** -8 + 2.0 ** -134
    return out, bound


@pytest.mark.parametrize("lens", [[333, 90], [5000, 1800]], ids=["whole", "cut"])
@pytest.mark.parametrize("N,G", [(1, 6), (9, 3), (16, 4), (35, 4)])
@pytest.mark.parametrize("d", [32, 64, 96, 160, 256])
def test_weights_hold_more_than_one_term(d, N, G, lens):
    c = AttnCase(2, 2 * G, 2, d, lens, N, random_tree, 64, seed=3)
    plan = plan_of(c.args.desc)
    print(form_of(c.args.desc, plan), segments_of(c.args.desc, plan, lens))
    c.run()
    torch.cuda.synchronize()
    got = f64(c.out)
    for b in range(2):
        want, bound = expected(f64(c.q[b]), *c.held(b), f64(c.k_tree[b]), f64(c.v_tree[b]), F.ancestors(c.parents[b]), c.scale)
        share = np.abs(got[b] - want) / bound
        assert share.max() <= 1, (b, float(share.max()), int((share > 1).sum()), share.size)
