"""Caches with sparse PSAC rows in windows of few Queries and in shared histories, against
the 64-bit softmax over the same tokens with a row in every slot."""
import numpy as np
import pytest
import torch

import oracle
import stream64 as s64
from paper_2609_26425_amd import quantwm as qw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Both(s64.Packed):
    """n tokens, four in five of them centroids (no residual, so no row), in a cache with a row
    a slot (cfg, cache) and in one with sparse rows (sparse_cfg, sparse_cache)."""

    def __init__(self, rng, batch, heads, d, r, dtype, starts, n):
        super().__init__(rng, batch, heads, d, 16, 32, r, dtype, 0, starts, n)
        more = dict(coef_stage=n)
        args = (batch, heads, d, 16, 32, r, 4, max(1, n))
        ocfg = oracle.cfg_of(*args, dtype == "bf16", qw.STORE_SPARSE, **more)
        self.sparse_cfg = qw.make_config(*args, dtype, qw.STORE_SPARSE, **more)
        self.cache, self.sparse_cache = oracle.new_cache(self.ocfg), oracle.new_cache(ocfg)
        for t, lo, hi in zip(self.tables, self.starts, self.starts[1:] + [n]):
            k, v = (s64.rounded(rng.standard_normal((batch, hi - lo, heads, d)), dtype) for _ in range(2))
            at = np.arange(hi - lo) % 5 != 0
            k[:, at] = np.asarray(t[0])[:, :, 3][:, None]
            for cfg, cache in ((self.ocfg, self.cache), (ocfg, self.sparse_cache)):
                oracle.append(cfg, t, cache, lo, k, v)

    def operands(self, sparse):
        cfg, cache = (self.sparse_cfg, self.sparse_cache) if sparse else (self.cfg, self.cache)
        return cfg, torch.from_numpy(cache).to(DEV)

    def sparse_blocks(self):
        """The calibration blocks do not depend on how rows are stored."""
        assert qw.quantwm_calib_bytes(self.cfg) == qw.quantwm_calib_bytes(self.sparse_cfg)
        return self.blocks()


@pytest.mark.parametrize("dtype,r,n_q", [("bf16", 8, 1), ("bf16", 13, 2), ("bf16", 32, 20), ("bf16", 8, 40), ("f32", 6, 1),
                                         ("f32", 16, 40)])
def test_window(dtype, r, n_q):
    rng, H, d, n, starts, n_sink, window = np.random.default_rng(r + n_q), 2, 64, 1500, [0, 100, 700], 40, 900
    p = Both(rng, 1, H, d, r, dtype, starts, n)
    q = s64.rounded(rng.standard_normal((1, n_q, H, d)), dtype)
    k, v = p.keys_values()
    hi = n - n_q + 1 + np.arange(n_q)[:, None]
    visible = (np.arange(n) < hi) & ((np.arange(n) < n_sink) | (np.arange(n) >= hi - window))
    ref = (*s64.softmax(p.logits(q), visible, v), s64.tolerances(q, k, n, r, dtype))  # the tiled kernel's form
    cfg, cache = p.operands(True)
    blocks, qd = p.sparse_blocks(), s64.dev(q, cfg.torch_dtype)
    for nb in (0, qw.quantwm_attend_window_workspace_bytes(cfg, n, 0, n_q, 1, n_sink, window)):
        ws = torch.empty(nb, dtype=torch.uint8, device=DEV) if nb else None
        out, lse = torch.full_like(qd, 7.0), torch.full((1, H, n_q), 7.0, device=DEV)
        qw.quantwm_attend_window(cfg, blocks, starts, cache, n, None, None, 0, qd, n_q, n - n_q, 1, n_sink, window, out, lse, ws)
        torch.cuda.synchronize()
        s64.check(out, lse, *ref)


@pytest.mark.parametrize("sparse_pre,sparse_own", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("dtype,r,n_q", [("bf16", 8, 1), ("bf16", 13, 3), ("bf16", 16, 60), ("f32", 8, 5)])
def test_shared(dtype, r, n_q, sparse_pre, sparse_own):
    B, H, d, n_pre, n_own, n_act = 3, 2, 64, 900, 200, 60
    rng = np.random.default_rng(r + n_q)
    pre, own = Both(rng, 1, H, d, r, dtype, [0, 300], n_pre), Both(rng, B, H, d, r, dtype, [0], n_own)
    q, ka, va = (s64.rounded(rng.standard_normal((B, m, H, d)), dtype) for m in (n_q, n_act, n_act))
    (pk, pv), (k, v), flat = pre.keys_values(), own.keys_values(), q.reshape(1, B * n_q, H, d)
    k, v = (np.concatenate([np.repeat(a, B, 0), b, x.transpose(0, 2, 1, 3)], 2) for a, b, x in ((pk, k, ka), (pv, v, va)))
    n = n_pre + n_own + n_act
    visible = np.arange(n) < (n - n_act + np.arange(n_q) + 1)[:, None]
    refs = []
    for few_pre in s64.forms(dtype)[:1 if sparse_pre else 2]:
        for few_own in s64.forms(dtype)[:1 if sparse_own else 2]:
            lg = np.concatenate([pre.logits(flat, few_pre).reshape(H, B, n_q, n_pre).transpose(1, 0, 2, 3),
                                 own.logits(q, few_own), s64.exact_logits(q, ka)], 3)
            res = np.concatenate([np.repeat(pre.residuals(), B, 0), own.residuals()], 2) if few_pre or few_own else None
            refs.append((*s64.softmax(lg, visible, v), s64.tolerances(q, k, 2 * n + 64, r, dtype, res)))
    (pcfg, pcache), (cfg, cache) = pre.operands(sparse_pre), own.operands(sparse_own)
    ws = torch.empty(qw.quantwm_attend_shared_workspace_bytes(pcfg, n_pre, cfg, n_own, n_act, n_q), dtype=torch.uint8, device=DEV)
    qd, kd, vd = (s64.dev(x, cfg.torch_dtype) for x in (q, ka, va))
    out, lse = torch.full_like(qd, 7.0), torch.empty(B, H, n_q, device=DEV)
    qw.quantwm_attend_shared(pcfg, pre.sparse_blocks(), pre.starts, pcache, n_pre, cfg, own.sparse_blocks(), cache, n_own, kd, vd,
                             n_act, qd, n_q, n - n_act, 1, out, lse, ws)
    torch.cuda.synchronize()
    s64.check_any(out, lse, refs)
