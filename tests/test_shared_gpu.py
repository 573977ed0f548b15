"""quantwm_attend_shared against a plain 64-bit softmax over [prefix | own packed | own
exact] keys: rollouts that do not fill a block of Queries, parts that are empty, a
prefix in epochs and in another format than the rollouts' caches, rows that see only
the prefix, one token each."""
import numpy as np
import pytest
import torch

import stream64 as s64
from paper_2609_26425_amd import quantwm as qw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# rollouts, heads, d, dtype, prefix (starts, n, centroids, group, rank, storage), own (packed, exact, centroids,
# group, rank, storage), frame, first own position of the Queries, Queries
CASES = {
    "tokens": (5, 2, 128, "bf16", ([0], 700, 32, 32, 8, 0), (30, 1, 16, 32, 8, 0), 1, 30, 1),
    "frames": (3, 2, 128, "bf16", ([0, 100, 300], 500, 37, 32, 16, 1), (130, 50, 16, 64, 4, 0), 50, 130, 100),
    "blocks": (3, 1, 128, "bf16", ([0], 300, 256, 64, 32, 0), (64, 300, 16, 32, 0, 1), 100, 64, 300),
    "prefix-only": (4, 2, 64, "bf16", ([0], 333, 16, 16, 4, 0), (0, 0, 16, 32, 8, 0), 1, 0, 7),
    "own-only": (2, 2, 128, "bf16", ([0], 0, 16, 32, 8, 0), (200, 20, 16, 32, 8, 0), 10, 190, 60),
    "no-keys": (2, 2, 128, "bf16", ([0], 0, 16, 32, 8, 0), (0, 0, 16, 32, 8, 0), 10, 0, 5),
    "one-rollout": (1, 2, 128, "bf16", ([0], 400, 16, 32, 8, 0), (70, 0, 16, 32, 8, 0), 1, 40, 30),
    "rows-before-own-keys": (2, 2, 128, "bf16", ([0], 400, 16, 32, 8, 0), (0, 90, 16, 32, 8, 0), 30, 0, 90),
    "one-prefix-key": (3, 2, 128, "bf16", ([0], 1, 16, 32, 8, 0), (0, 3, 16, 32, 8, 0), 1, 0, 3),
    "long-prefix": (16, 2, 64, "bf16", ([0, 5000], 9000, 64, 32, 8, 0), (20, 0, 16, 32, 8, 0), 1, 20, 2),
    "few-frames": (3, 2, 128, "bf16", ([0, 100, 300], 8000, 64, 16, 12, 1), (200, 40, 100, 64, 32, 0), 2, 220, 7),
    "few-own": (30, 2, 64, "bf16", ([0], 12_000, 64, 32, 16, 0), (100, 1, 16, 32, 8, 1), 1, 100, 1),
    "few-own-wide": (2, 2, 128, "bf16", ([0], 500, 200, 32, 16, 0), (400, 1, 250, 32, 32, 1), 1, 300, 1),
    "f32": (3, 2, 64, "f32", ([0, 99], 700, 16, 32, 4, 0), (70, 33, 16, 32, 4, 0), 1, 70, 33),
    "f32-128": (2, 2, 128, "f32", ([0], 200, 16, 32, 32, 1), (65, 0, 16, 16, 8, 0), 20, 45, 40),
    # more heads than CUs: parts in the order of their segments
    "many-rollouts": (70, 4, 64, "bf16", ([0, 64], 150, 16, 32, 8, 0), (40, 3, 16, 32, 4, 0), 1, 41, 2),
    "f32-many-rollouts": (40, 8, 64, "f32", ([0, 64], 150, 16, 32, 8, 0), (40, 3, 16, 32, 4, 0), 1, 41, 2),
    # fp32 passes that share a grid, in two formats, and that do not (ranks, scales)
    "f32-two-formats": (4, 3, 64, "f32", ([0, 64, 200], 333, 37, 16, 12, 0), (130, 5, 8, 64, 3, 0), 2, 100, 9),
    "f32-i8": (2, 2, 128, "f32", ([0], 300, 64, 32, 8, 1), (90, 0, 16, 16, 16, 1), 1, 60, 40),
    "f32-ranks-apart": (2, 2, 64, "f32", ([0], 300, 16, 32, 20, 0), (90, 7, 16, 16, 0, 0), 1, 60, 40),
    "f32-scales-apart": (2, 2, 64, "f32", ([0], 300, 16, 32, 8, 0), (90, 7, 16, 16, 8, 1), 1, 60, 40),
}


@pytest.mark.parametrize("name", list(CASES))
def test_shared(name):
    B, H, d, dtype, (starts, n_pre, *pfmt), (n_pk, n_act, *fmt), frame, first, n_q = CASES[name]
    rng = np.random.default_rng(B + n_pre + d)
    pkc, pg, pr, pst = pfmt
    kc, g, r, st = fmt
    pre = s64.Packed(rng, 1, H, d, pkc, pg, pr, dtype, pst, starts, n_pre)
    own = s64.Packed(rng, B, H, d, kc, g, r, dtype, st, [0], n_pk)
    q = s64.rounded(rng.standard_normal((B, n_q, H, d)), dtype)
    pk, pv = pre.keys_values()
    k, v = own.keys_values()
    flat = q.reshape(1, B * n_q, H, d)
    ka = va = None
    if n_act:
        ka, va = (s64.rounded(rng.standard_normal((B, n_act, H, d)), dtype) for _ in range(2))
        k, v = (np.concatenate([x, y.transpose(0, 2, 1, 3)], 2) for x, y in ((k, ka), (v, va)))
    k, v = (np.concatenate([np.repeat(x, B, 0), y], 2) for x, y in ((pk, k), (pv, v)))
    n, q_start = n_pre + n_pk + n_act, n_pre + first
    visible = np.arange(n) < (q_start + (np.arange(n_q) // frame + 1) * frame)[:, None]
    refs = []
    for few_pre in s64.forms(dtype):
        for few_own in s64.forms(dtype):
            parts = [pre.logits(flat, few_pre).reshape(H, B, n_q, n_pre).transpose(1, 0, 2, 3), own.logits(q, few_own)]
            if n_act:
                parts.append(s64.exact_logits(q, ka))
            # the join adds the weights of the parts: n 2^-24 more covers its exponentials and sums
            tol = [max(x) for x in zip(
                s64.tolerances(q, k, 2 * n + 64, max(r, pr), dtype, own.residuals() if few_own else None),
                s64.tolerances(flat, pk, 2 * n + 64, max(r, pr), dtype, pre.residuals() if few_pre else None))]
            refs.append((*s64.softmax(np.concatenate(parts, 3), visible, v), tol))
    dt = own.cfg.torch_dtype
    nb = qw.quantwm_attend_shared_workspace_bytes(pre.cfg, n_pre, own.cfg, n_pk, n_act, n_q)
    assert (nb > 0) == (n > 0)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV) if nb else None
    qd, (kd, vd) = s64.dev(q, dt), (s64.dev(ka, dt), s64.dev(va, dt)) if n_act else (None, None)
    # the pointers of an empty part are not read
    pb, pc = (pre.blocks(), pre.on_device()) if n_pre else (None, None)
    ob, oc = (own.blocks(), own.on_device()) if n_pk + n_act else (None, None)
    for with_lse in (True, False):
        out, lse = torch.full_like(qd, 7.0), torch.full((B, H, n_q), 7.0, device=DEV)
        qw.quantwm_attend_shared(pre.cfg, pb, starts, pc, n_pre, own.cfg, ob, oc, n_pk, kd, vd, n_act, qd, n_q, q_start,
                                 frame, out, lse if with_lse else None, ws)
        torch.cuda.synchronize()
        if with_lse:
            s64.check_any(out, lse, refs)
            first_out = out
        else:
            assert torch.equal(out, first_out)
