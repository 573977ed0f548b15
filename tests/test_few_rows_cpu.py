"""Which kernel a call takes, from the workspace it asks for: the few-row kernels hold 16
partial planes and one more at least, the tiles at most 16. No kernel is launched."""
import pytest

from paper_2609_26425_amd import quantwm as qw


def _cfg(dtype="bf16", batch=1, heads=40, d=128, rank=16, storage=0):
    return qw.make_config(batch, heads, d, 128, 32, rank, 4, 1 << 20, dtype, storage, coef_stage=64 if storage & 4 else 0)


def _planes(nb, cfg, n_q):
    return nb // (cfg.batch * cfg.heads * n_q * (cfg.head_dim * 4 + 8))


# heads, Queries, keys, window (None: all), config: whether the few-row kernel takes it
CALLS = {
    "one": (True, 40, 1, 32_760, 15_600, {}), "one-i8": (True, 40, 1, 32_760, None, dict(storage=1)),
    "rank-0": (True, 12, 1, 900, None, dict(rank=0)), "odd-rank": (False, 40, 1, 32_760, 15_600, dict(rank=13)),
    "rank-6": (False, 40, 1, 32_760, 15_600, dict(rank=6)), "sparse": (False, 40, 1, 32_760, 15_600, dict(storage=4)),
    "sixteen": (True, 12, 16, 5760, None, {}), "sixteen-of-fewer": (False, 12, 16, 5759, None, {}),
    "sixteen-windowed": (False, 12, 16, 100_000, 5000, {}), "block": (True, 12, 32, 11_904, None, {}),
    "two-blocks": (False, 12, 33, 100_000, None, {}),
    "f32": (True, 2, 257, 362, None, dict(dtype="f32", d=64, rank=4)),
    "f32-odd-rank": (True, 2, 257, 362, None, dict(dtype="f32", d=64, rank=13)),
    "f32-sparse": (False, 2, 257, 362, None, dict(dtype="f32", d=64, rank=4, storage=4)),
    "f32-many": (False, 30, 128, 10_000, None, dict(dtype="f32")),
    "f32-many-windowed": (True, 30, 128, 10_000, 1500, dict(dtype="f32")),
    "f32-long": (False, 1, 4097, 1000, None, dict(dtype="f32")),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_window(name):
    few, heads, n_q, n, window, kw = CALLS[name]
    cfg = _cfg(heads=heads, **kw)
    nb = qw.quantwm_attend_window_workspace_bytes(cfg, n, 0, n_q, 1, 0, n if window is None else window)
    assert (_planes(nb, cfg, n_q) > 16) == few


@pytest.mark.parametrize("n_pre,n_own,n_q,kw,few_pre,few_own", [
    (24_960, 131, 1, {}, True, True), (24_960, 131, 3, {}, False, False), (24_960, 800, 2, {}, True, True),
    (24_960, 800, 2, dict(rank=13), False, False), (24_960, 800, 1, dict(storage=4), False, False),
    (777, 103, 33, dict(dtype="f32", heads=2, d=64, rank=4), True, True),
    (777, 103, 33, dict(dtype="f32", heads=2, d=64, rank=4, storage=4), False, False),
])
def test_shared(n_pre, n_own, n_q, kw, few_pre, few_own):
    """16 rollouts, whose rows are one chunk to the prefix; each part by itself."""
    pre, own = _cfg(**{"heads": 30, **kw}), _cfg(batch=16, **{"heads": 30, **kw})
    size = qw.quantwm_attend_shared_workspace_bytes
    assert (_planes(size(pre, n_pre, own, 0, 0, n_q), own, n_q) > 16) == few_pre
    assert (_planes(size(pre, 0, own, n_own, 0, n_q), own, n_q) > 16) == few_own
