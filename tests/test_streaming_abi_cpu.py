"""Host-side checks of the windowed, shared and rotary entry points: what they refuse,
before anything is enqueued, and their size queries. No kernel is launched."""
import ctypes

import pytest
import torch

from paper_2609_26425_amd import quantwm as qw

P = ctypes.c_void_p
A, B_, C_, D_, E_, F_ = (P(i * 0x10000000) for i in range(1, 7))  # far apart, aligned, never read
CFG = dict(batch=1, heads=2, head_dim=128, n_centroids=16, group_size=32, rank=8, top_m=4, capacity=1000, dtype="bf16")


def _cfg(**kw):
    return qw.make_config(**{**CFG, **kw})


def _window(cfg=None, **kw):
    a = dict(calib=A, n_epochs=1, starts=None, cache=B_, n_cache=500, ka=None, va=None, n_act=0, q=C_, n_q=10,
             q_start=490, frame=1, n_sink=0, window=100, out=D_, lse=None, ws=None, nb=0)
    a.update(kw)
    return qw.library().quantwm_attend_window(
        ctypes.byref(cfg or _cfg()), a["calib"], a["n_epochs"], a["starts"], a["cache"], a["n_cache"], a["ka"], a["va"],
        a["n_act"], a["q"], a["n_q"], a["q_start"], a["frame"], a["n_sink"], a["window"], a["out"], a["lse"], a["ws"],
        a["nb"], None)


def _starts(*x):
    return (ctypes.c_int64 * len(x))(*x)


@pytest.mark.parametrize("kw,status,word", [
    (dict(n_sink=-1), qw.ERR_INVALID_ARG, "n_sink"), (dict(window=-5), qw.ERR_INVALID_ARG, "window"),
    (dict(n_cache=1001, q_start=0), qw.ERR_CAPACITY, "capacity"), (dict(n_cache=-1), qw.ERR_INVALID_ARG, "sizes"),
    (dict(q_start=501), qw.ERR_INVALID_ARG, "q_start"), (dict(frame=0), qw.ERR_INVALID_ARG, "frame_tokens"),
    (dict(n_epochs=0), qw.ERR_UNSUPPORTED, "n_epochs"), (dict(n_epochs=65), qw.ERR_UNSUPPORTED, "n_epochs"),
    (dict(n_epochs=2), qw.ERR_INVALID_ARG, "epoch_start"),
    (dict(n_epochs=2, starts=_starts(0, 63)), qw.ERR_INVALID_ARG, "64"),
    (dict(n_epochs=2, starts=_starts(0, 500)), qw.ERR_INVALID_ARG, "n_cache"),
    (dict(calib=None), qw.ERR_INVALID_ARG, "calib"), (dict(cache=None), qw.ERR_INVALID_ARG, "cache"),
    (dict(q=P(0x1008)), qw.ERR_INVALID_ARG, "q is not"), (dict(out=None), qw.ERR_INVALID_ARG, "out"),
    (dict(lse=P(0x1002)), qw.ERR_INVALID_ARG, "lse"), (dict(n_act=5), qw.ERR_INVALID_ARG, "k_act"),
    (dict(ws=P(0x1010), nb=1 << 20), qw.ERR_INVALID_ARG, "256"),
    (dict(n_q=0x7fff0001), qw.ERR_UNSUPPORTED, "Queries"),
])
def test_window_refuses(kw, status, word):
    assert _window(**kw) == status
    assert word in qw.quantwm_last_error()


def test_window_sizes():
    cfg = _cfg(capacity=1 << 20)
    ws = qw.quantwm_attend_window_workspace_bytes
    assert _window(n_q=0) == qw.OK  # no Queries: nothing to do
    # the split goes by the keys in reach, not by the cache
    assert ws(cfg, 1 << 20, 0, 100, 1, 64, 1000) == ws(cfg, 1 << 18, 0, 100, 1, 64, 1000)
    assert ws(cfg, 1 << 20, 0, 100, 1, 0, 1 << 62) == qw.quantwm_attend_workspace_bytes(cfg, 1 << 20, 100)
    assert ws(cfg, 1 << 20, 0, 100, 1, 1 << 62, 0) == qw.quantwm_attend_workspace_bytes(cfg, 1 << 20, 100)
    assert ws(cfg, 1 << 20, 0, 100, 1 << 30, 0, 10) == qw.quantwm_attend_workspace_bytes(cfg, 1 << 20, 100)
    for bad in ((-1, 0, 100, 1, 0, 10), (100, -1, 100, 1, 0, 10), (100, 0, 0, 1, 0, 10), (100, 0, 10, 0, 0, 10),
                (100, 0, 10, 1, -1, 10), (100, 0, 10, 1, 0, -1)):
        assert ws(cfg, *bad) == 0


def _shared(pcfg=None, cfg=None, **kw):
    a = dict(pcalibs=A, n_epochs=1, starts=None, pcache=B_, n_prefix=500, calib=A, cache=C_, n_cache=100, ka=None,
             va=None, n_act=0, q=D_, n_q=4, q_start=596, frame=1, out=E_, lse=None, ws=F_, nb=1 << 40)
    a.update(kw)
    return qw.library().quantwm_attend_shared(
        ctypes.byref(pcfg or _cfg()), a["pcalibs"], a["n_epochs"], a["starts"], a["pcache"], a["n_prefix"],
        ctypes.byref(cfg or _cfg(batch=3)), a["calib"], a["cache"], a["n_cache"], a["ka"], a["va"], a["n_act"], a["q"],
        a["n_q"], a["q_start"], a["frame"], a["out"], a["lse"], a["ws"], a["nb"], None)


@pytest.mark.parametrize("kw,status,word", [
    (dict(pcfg=_cfg(batch=2)), qw.ERR_INVALID_ARG, "batch 1"), (dict(pcfg=_cfg(heads=3)), qw.ERR_INVALID_ARG, "agree"),
    (dict(pcfg=_cfg(head_dim=64)), qw.ERR_INVALID_ARG, "agree"), (dict(pcfg=_cfg(dtype="f32")), qw.ERR_INVALID_ARG, "agree"),
    (dict(cfg=_cfg(rank=33)), qw.ERR_UNSUPPORTED, "rank"), (dict(q_start=499), qw.ERR_INVALID_ARG, "q_start"),
    (dict(q_start=601), qw.ERR_INVALID_ARG, "q_start"), (dict(n_prefix=1001, q_start=1001), qw.ERR_CAPACITY, "capacity"),
    (dict(n_cache=1001), qw.ERR_CAPACITY, "capacity"), (dict(n_prefix=-1), qw.ERR_INVALID_ARG, "sizes"),
    (dict(n_q=0x7fff0000 // 3 + 1), qw.ERR_UNSUPPORTED, "Queries"), (dict(frame=0), qw.ERR_INVALID_ARG, "frame_tokens"),
    (dict(n_epochs=2, starts=_starts(0, 10)), qw.ERR_INVALID_ARG, "64"),
    (dict(pcalibs=None), qw.ERR_INVALID_ARG, "prefix_calibs"), (dict(pcache=None), qw.ERR_INVALID_ARG, "prefix_cache"),
    (dict(calib=None), qw.ERR_INVALID_ARG, "calib"), (dict(cache=P(0x8)), qw.ERR_INVALID_ARG, "cache"),
    (dict(n_act=2), qw.ERR_INVALID_ARG, "k_act"), (dict(q=None), qw.ERR_INVALID_ARG, "q is null"),
    (dict(out=None), qw.ERR_INVALID_ARG, "out"), (dict(lse=P(2)), qw.ERR_INVALID_ARG, "lse"),
    (dict(ws=None, nb=0), qw.ERR_INVALID_ARG, "workspace"), (dict(ws=P(0x1010)), qw.ERR_INVALID_ARG, "256"),
    (dict(nb=100), qw.ERR_INVALID_ARG, "too small"),
])
def test_shared_refuses(kw, status, word):
    assert _shared(**kw) == status
    assert word in qw.quantwm_last_error()


def test_shared_sizes():
    pcfg, cfg = _cfg(capacity=1 << 20), _cfg(batch=3)
    ws = qw.quantwm_attend_shared_workspace_bytes
    assert _shared(n_q=0) == qw.OK
    up = lambda x: (x + 255) // 256 * 256  # noqa: E731
    rows = 3 * 2 * 4  # of one plane: running maxima, sums and 128 channels each
    prefix, mine = ws(pcfg, 64, cfg, 0, 0, 4), ws(pcfg, 0, cfg, 64, 0, 4)
    assert prefix >= rows * 130 * 4 and mine >= rows * 130 * 4 and prefix % 256 == 0
    assert ws(pcfg, 64, cfg, 64, 0, 4) == prefix + mine == ws(pcfg, 64, cfg, 60, 4, 4)
    # many rows: one plane a part once the launch fills the GPU
    big = 3 * 2 * 50_000
    assert ws(pcfg, 64, cfg, 0, 0, 50_000) == up(up(big * 128 * 4) + big * 8)
    assert ws(pcfg, 0, cfg, 0, 0, 4) == ws(pcfg, 64, cfg, 64, 0, 0) == 0
    assert ws(_cfg(batch=2), 64, cfg, 64, 0, 4) == 0 and ws(pcfg, -1, cfg, 64, 0, 4) == 0


def _axes(**kw):
    a = qw.RotaryAxes()
    a.pairs, a.height, a.width = kw.get("pairs", 0), kw.get("height", 4), kw.get("width", 5)
    for i, x in enumerate(kw.get("dims", (44, 42, 42))):
        a.dims[i] = x
    for i in range(64):
        a.freq[i] = kw.get("freq", 0.5)
    return a


def _rotary(cfg=None, axes=None, **kw):
    a = dict(pos0=0, pos=None, q=A, k=B_, n=7, stride=256, qo=C_, ko=D_, inverse=0)
    a.update(kw)
    return qw.library().quantwm_rotary(ctypes.byref(cfg or _cfg()), ctypes.byref(axes or _axes()), a["pos0"], a["pos"],
                                       a["q"], a["k"], a["n"], a["stride"], a["qo"], a["ko"], a["inverse"], None)


BYTES = 7 * 256 * 2  # of one tensor in _rotary


@pytest.mark.parametrize("kw,status,word", [
    (dict(axes=_axes(pairs=2)), qw.ERR_INVALID_ARG, "pairs"), (dict(axes=_axes(dims=(43, 42, 42))), qw.ERR_INVALID_ARG, "even"),
    (dict(axes=_axes(dims=(-2, 42, 42))), qw.ERR_INVALID_ARG, "even"), (dict(axes=_axes(dims=(64, 64, 2))), qw.ERR_INVALID_ARG, "sum"),
    (dict(axes=_axes(pairs=1, dims=(20, 20, 20))), qw.ERR_UNSUPPORTED, "16"),
    (dict(axes=_axes(freq=float("nan"))), qw.ERR_INVALID_ARG, "freq"), (dict(n=-1), qw.ERR_INVALID_ARG, "n must"),
    (dict(axes=_axes(height=0)), qw.ERR_INVALID_ARG, "height"), (dict(pos0=-1), qw.ERR_INVALID_ARG, "positions"),
    (dict(pos0=20 << 31), qw.ERR_INVALID_ARG, "positions"), (dict(pos0=1 << 62), qw.ERR_INVALID_ARG, "positions"),
    (dict(q=None), qw.ERR_INVALID_ARG, "q is null"), (dict(qo=None), qw.ERR_INVALID_ARG, "q_out"),
    (dict(k=None), qw.ERR_INVALID_ARG, "together"), (dict(ko=None), qw.ERR_INVALID_ARG, "together"),
    (dict(k=P(0x1004)), qw.ERR_INVALID_ARG, "k is not"), (dict(stride=255), qw.ERR_INVALID_ARG, "token_stride"),
    (dict(stride=260), qw.ERR_INVALID_ARG, "token_stride"), (dict(pos=P(0x90000002)), qw.ERR_INVALID_ARG, "pos"),
    (dict(n=0x7fff0001), qw.ERR_UNSUPPORTED, "tokens"),
    # overlaps: shifted, strided in place, crossed, outputs of one another, positions
    (dict(qo=P(A.value + 512)), qw.ERR_INVALID_ARG, "overlap"), (dict(stride=512, qo=A), qw.ERR_INVALID_ARG, "overlap"),
    (dict(qo=B_, ko=C_), qw.ERR_INVALID_ARG, "overlap"), (dict(ko=P(C_.value + BYTES - 16)), qw.ERR_INVALID_ARG, "overlap"),
    (dict(pos=P(C_.value + BYTES - 4)), qw.ERR_INVALID_ARG, "overlap"),
])
def test_rotary_refuses(kw, status, word):
    assert _rotary(**kw) == status
    assert word in qw.quantwm_last_error()


def test_rotary_axes():
    cfg = _cfg()
    assert _rotary(n=0) == qw.OK
    a = qw.rotary_axes(cfg, (44, 42, 42), 30, 52)
    assert (a.height, a.width, a.pairs, list(a.dims)) == (30, 52, 0, [44, 42, 42])
    want = [1e4 ** (-2 * i / D) for D in (44, 42, 42) for i in range(D // 2)]
    assert list(a.freq) == pytest.approx(want, rel=1e-15)
    for dims in ((3, 2, 2), (64, 64, 2), (-2, 4, 4)):
        with pytest.raises(qw.QuantwmError):
            qw.rotary_axes(cfg, dims, 4, 5)
    with pytest.raises(qw.QuantwmError, match="pairs"):
        qw.rotary_axes(cfg, (44, 42, 42), 4, 5, pairs=2)
    for base in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(qw.QuantwmError):
            qw.rotary_axes(cfg, (44, 42, 42), 4, 5, base=base)
    with pytest.raises(ValueError):
        qw.rotary_axes(cfg, (44, 42, 42), 4, 5, freq=[1.0])


def test_the_binding_refuses_tensors_that_do_not_fit():
    cfg = _cfg(batch=2)
    axes = qw.rotary_axes(cfg, (44, 42, 42), 4, 5)
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)  # noqa: E731
    x, out = z(2, 7, 2, 128), z(2, 7, 2, 128)
    for args in [(z(2, 7, 2, 128, dt=torch.float32), out), (z(2, 6, 2, 128), out), (x, z(2, 6, 2, 128)),
                 (z(2, 7, 128, 2).transpose(2, 3), out), (z(7, 2, 2, 128).transpose(0, 1), out),
                 (z(2, 9, 2, 128)[:, 1:8], out)]:
        with pytest.raises(ValueError):
            qw.quantwm_rotary(cfg, axes, args[0], None, 7, args[1])
    with pytest.raises(ValueError):
        qw.quantwm_rotary(cfg, axes, x, None, 7, out, pos=z(2, 7, 3, dt=torch.int64))
    calib, cache = z(qw.quantwm_calib_bytes(cfg), dt=torch.uint8), z(qw.quantwm_cache_bytes(cfg), dt=torch.uint8)
    good = dict(cfg=cfg, calibs=calib, epoch_start=[0], cache=cache, n_cache=100, k_act=x, v_act=x, n_act=7, q=x, n_q=7,
                q_start=100, frame_tokens=1, n_sink=0, window=10, out=out)
    for bad in (dict(calibs=calib[:-1]), dict(cache=cache[:-1]), dict(k_act=x[:1]), dict(v_act=x.float()), dict(q=x[:1]),
                dict(out=out[:1]), dict(lse_out=z(2, 2, 7)), dict(lse_out=z(2, 2, 6, dt=torch.float32)),
                dict(epoch_start=[0, 64])):
        with pytest.raises(ValueError):
            qw.quantwm_attend_window(**{**good, **bad})
    pcfg = _cfg()
    pcalib, pcache = z(qw.quantwm_calib_bytes(pcfg), dt=torch.uint8), z(qw.quantwm_cache_bytes(pcfg), dt=torch.uint8)
    good = dict(prefix_cfg=pcfg, prefix_calibs=pcalib, epoch_start=[0], prefix_cache=pcache, n_prefix=100, cfg=cfg,
                calib=calib, cache=cache, n_cache=100, k_act=x, v_act=x, n_act=7, q=x, n_q=7, q_start=200, frame_tokens=1,
                out=out)
    for bad in (dict(prefix_calibs=pcalib[:-1]), dict(prefix_cache=pcache[:-1]), dict(calib=calib[:-1]), dict(q=x[:1])):
        with pytest.raises(ValueError):
            qw.quantwm_attend_shared(**{**good, **bad})


def test_window_without_keys_over_many_blocks():
    """512 rollouts of 4,096 fp32 Queries are more blocks of 32 than a grid dimension has,
    whether they see keys or not: they take blocks of 256, unsplit."""
    lib = qw.library()
    cfg = _cfg(batch=512, dtype="f32")
    for n_cache in (0, 64):
        assert lib.quantwm_attend_window_workspace_bytes(ctypes.byref(cfg), n_cache, 0, 4096, 1, 0, 16) == 0
    # nor are more heads taken than one dimension has room for, in parts
    many = _cfg(batch=40_000)
    assert lib.quantwm_attend_window_workspace_bytes(ctypes.byref(many), 64, 0, 1, 1, 0, 16) == 0


@pytest.mark.parametrize("kw,word", [
    # an angle past the doubles, for positions below 2^31; a stride whose bytes pass 64 bits
    (dict(axes=_axes(freq=1e300)), "freq"), (dict(n=0x7fff0000, stride=1 << 40), "stride"),
])
def test_rotary_refuses_what_overflows(kw, word):
    assert _rotary(**kw) == qw.ERR_INVALID_ARG
    assert word in qw.quantwm_last_error()


def test_rotary_refuses_rows_past_its_counters():
    assert _rotary(cfg=_cfg(heads=1 << 24), n=1, stride=1 << 31) == qw.ERR_UNSUPPORTED
    assert "2^30" in qw.quantwm_last_error()
