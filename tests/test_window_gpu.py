"""quantwm_attend_window against a plain 64-bit softmax, at the bounds where a window
goes wrong: sinks and windows that end inside tiles, on them, inside another epoch or
inside the exact chunk, rows that see nothing, holes of one tile and of whole epochs,
key splits, one Query. Most Queries put their weight on a key at a bound of their own
mask (the first and last visible ones and their neighbours outside)."""
import numpy as np
import pytest
import torch

import oracle
import stream64 as s64
from paper_2609_26425_amd import quantwm as qw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# batch, starts, packed, exact, storage, d, centroids, rank, group, frame, n_sink, window, q_start, n_q, dtype
CASES = {
    "causal": (1, [0], 700, 0, 0, 128, 16, 8, 32, 1, 5, 130, 410, 290, "bf16"),
    "causal-act": (1, [0], 500, 77, 1, 128, 16, 8, 32, 1, 70, 64, 300, 277, "bf16"),
    "frames": (2, [0, 200, 500], 900, 100, 0, 128, 37, 12, 32, 50, 50, 150, 700, 300, "bf16"),
    "frames-i8": (1, [0, 64, 128, 192], 640, 0, 1, 64, 16, 16, 16, 30, 30, 90, 350, 290, "bf16"),
    "one-query": (1, [0], 3000, 0, 0, 128, 64, 16, 32, 1, 100, 1000, 2999, 1, "bf16"),
    "one-key": (1, [0], 1, 0, 0, 128, 4, 8, 32, 1, 0, 1, 0, 1, "bf16"),
    "itself-only": (1, [0], 300, 0, 0, 128, 16, 8, 32, 1, 0, 1, 0, 300, "bf16"),
    "sinks-only": (1, [0], 700, 0, 0, 128, 16, 8, 32, 1, 65, 0, 400, 300, "bf16"),
    "nothing": (1, [0], 700, 30, 0, 128, 16, 8, 32, 1, 0, 0, 400, 300, "bf16"),
    "past-the-keys": (1, [0], 300, 0, 0, 128, 16, 8, 32, 1, 0, 40, 290, 200, "bf16"),
    "past-with-sinks": (1, [0], 300, 10, 0, 64, 16, 0, 32, 7, 3, 40, 300, 300, "bf16"),
    "everything": (1, [0, 300], 700, 50, 0, 128, 16, 8, 32, 25, 0, 1 << 62, 450, 300, "bf16"),
    "all-sinks": (1, [0], 700, 50, 0, 128, 16, 8, 32, 25, 1 << 62, 0, 450, 300, "bf16"),
    "tile-bounds": (1, [0, 320], 1024, 0, 0, 128, 16, 8, 32, 64, 64, 128, 768, 256, "bf16"),
    "hole-of-a-tile": (1, [0], 512, 0, 0, 128, 16, 8, 32, 32, 64, 384, 480, 32, "bf16"),
    "epochs-in-the-hole": (1, [0, 100, 200, 300, 900], 1300, 0, 0, 128, 16, 8, 32, 10, 20, 150, 1100, 200, "bf16"),
    "packed-in-the-hole": (1, [0], 300, 900, 0, 128, 16, 8, 32, 1, 0, 100, 900, 300, "bf16"),
    "sinks-in-the-chunk": (1, [0], 64, 900, 1, 128, 16, 8, 32, 1, 100, 100, 700, 264, "bf16"),
    "chunk-only": (1, [0], 0, 700, 0, 128, 16, 8, 32, 20, 30, 100, 400, 300, "bf16"),
    "first-rows": (1, [0], 256, 44, 0, 128, 16, 8, 32, 1, 2, 50, 0, 300, "bf16"),
    "no-tables": (1, [0, 400], 900, 60, 0, 128, 256, 32, 64, 20, 20, 200, 660, 300, "bf16"),
    "split": (2, [0, 3000], 6000, 100, 0, 64, 16, 8, 32, 20, 500, 2500, 6000, 100, "bf16"),
    "f32": (1, [0, 100, 500], 1090, 129, 0, 64, 16, 4, 32, 50, 60, 300, 919, 290, "f32"),
    "f32-i8-128": (2, [0], 600, 0, 1, 128, 16, 32, 16, 1, 7, 200, 400, 200, "f32"),
    "f32-nothing": (1, [0], 200, 0, 0, 64, 16, 0, 32, 1, 0, 10, 190, 60, "f32"),
}


def _bounds(q_start, n_q, frame, n_sink, window, n):
    hi = q_start + (np.arange(n_q) // frame + 1) * frame
    j = np.arange(n)
    visible = (j < hi[:, None]) & ((j < n_sink) | (j >= hi[:, None] - window))
    return hi, visible


# the same with few Queries, where another kernel runs; first its own shapes: group sizes
# against a lane's channels, ranks that are no multiple of four, many parts
FEW = {
    "g16": (2, [0], 2600, 40, 0, 128, 16, 12, 16, 1, 40, 2400, 2620, 7, "bf16"),
    "g16-i8": (1, [0, 333], 6200, 0, 1, 128, 100, 16, 16, 1, 40, 5900, 6150, 16, "bf16"),
    "g16-i8-32": (1, [0, 333], 12_000, 0, 1, 128, 100, 16, 16, 5, 11_990, 40, 11_950, 32, "bf16"),
    "g32-i8-25": (1, [0], 9400, 30, 1, 128, 128, 32, 32, 1, 300, 9100, 9400, 25, "bf16"),
    "g64": (1, [0], 7400, 31, 0, 64, 16, 8, 64, 3, 40, 7400, 7400, 20, "bf16"),
    "g64-i8": (1, [0], 12_000, 33, 1, 64, 256, 28, 64, 3, 13_000, 0, 11_990, 32, "bf16"),
    "g64-128": (1, [0], 6700, 10, 0, 128, 60, 32, 64, 2, 10, 6600, 6690, 18, "bf16"),
    "g32-64": (1, [0, 64, 200, 3000], 6400, 0, 1, 64, 200, 20, 32, 1, 0, 1 << 50, 6380, 17, "bf16"),
    "g16-64": (2, [0], 2000, 0, 0, 64, 30, 4, 16, 1, 33, 1900, 1990, 6, "bf16"),
    "g16-64-20": (1, [0], 7400, 0, 0, 64, 30, 4, 16, 20, 33, 7300, 7380, 20, "bf16"),
    "rank-0-20": (1, [0], 7400, 5, 0, 128, 30, 0, 32, 1, 33, 7300, 7380, 20, "bf16"),
    "odd-rank": (1, [0], 4000, 10, 0, 128, 60, 13, 32, 2, 10, 3900, 3990, 10, "bf16"),
    "many-epochs": (1, [66 * i for i in range(40)], 2700, 20, 0, 64, 8, 4, 16, 5, 70, 2600, 2600, 7, "bf16"),
    "many-epochs-19": (1, [180 * i for i in range(40)], 7200, 20, 0, 64, 8, 4, 16, 5, 70, 7100, 7200, 19, "bf16"),
    "early-rows": (1, [0], 7400, 0, 0, 128, 200, 16, 32, 1, 4, 7400, 0, 20, "bf16"),
    "early-row": (1, [0], 7400, 0, 1, 128, 200, 16, 32, 1, 4, 7400, 100, 1, "bf16"),
    "past-the-keys-few": (1, [0], 4000, 20, 0, 128, 32, 8, 32, 1, 0, 3900, 4020, 6, "bf16"),
    "long": (1, [0], 30_000, 100, 0, 64, 32, 8, 32, 1, 500, 20_000, 30_050, 3, "bf16"),
}
SHORT = {f"{k}-{m}": v[:13] + (m, v[14]) for k, v in CASES.items() if v[14] == "bf16" and v[13] > 2 for m in (1, 2)}


@pytest.mark.parametrize("name", list(CASES) + list(FEW) + list(SHORT))
def test_window(name):
    B, starts, n_pk, n_act, st, d, kc, r, g, frame, n_sink, window, q_start, n_q, dtype = \
        {**CASES, **FEW, **SHORT}[name]
    H, n = 2, n_pk + n_act
    rng = np.random.default_rng(n + d + n_sink % 1000)
    p = s64.Packed(rng, B, H, d, kc, g, r, dtype, st, starts, n_pk)
    k, v = p.keys_values()
    ka = va = None
    if n_act:
        ka, va = (s64.rounded(rng.standard_normal((B, n_act, H, d)), dtype) for _ in range(2))
        k, v = (np.concatenate([x, y.transpose(0, 2, 1, 3)], 2) for x, y in ((k, ka), (v, va)))
    hi, visible = _bounds(q_start, n_q, frame, n_sink, window, n)
    q = 0.5 * rng.standard_normal((B, n_q, H, d))
    for i in range(n_q):
        at = [hi[i] - 1, hi[i], hi[i] - window, hi[i] - window - 1, n_sink - 1, n_sink, None][i % 7]
        if at is not None:  # about 25 above the other logits at d = 128
            q[:, i] += 2.0 * k[:, :, min(max(at, 0), n - 1)]
    q = s64.rounded(q, dtype)
    refs = []
    for few in s64.forms(dtype):
        logits = p.logits(q, few)
        if n_act:
            logits = np.concatenate([logits, s64.exact_logits(q, ka)], 3)
        refs.append((*s64.softmax(logits, visible, v), s64.tolerances(q, k, n, r, dtype, p.residuals() if few else None)))
    dt = p.cfg.torch_dtype
    calibs, cache, qd = p.blocks(), p.on_device(), s64.dev(q, dt)
    kd, vd = (s64.dev(ka, dt), s64.dev(va, dt)) if n_act else (None, None)
    most = qw.quantwm_attend_window_workspace_bytes(p.cfg, n_pk, n_act, n_q, frame, n_sink, window)
    assert (name != "split") or most > 0
    for nb in sorted({0, most, most // 2}):
        ws = torch.empty(nb, dtype=torch.uint8, device=DEV) if nb else None
        out, lse = torch.full_like(qd, 7.0), torch.full((B, H, n_q), 7.0, device=DEV)
        qw.quantwm_attend_window(p.cfg, calibs, p.starts, cache, n_pk, kd, vd, n_act, qd, n_q, q_start, frame, n_sink,
                                 window, out, lse, ws)
        torch.cuda.synchronize()
        s64.check_any(out, lse, refs)
        only = torch.full_like(qd, 7.0)  # without the log-sum-exp
        qw.quantwm_attend_window(p.cfg, calibs, p.starts, cache, n_pk, kd, vd, n_act, qd, n_q, q_start, frame, n_sink,
                                 window, only, None, ws)
        assert torch.equal(only, out)


def _random(cfg, n, gen):
    return torch.randn(cfg.batch, n, cfg.heads, cfg.head_dim, generator=gen, device=DEV).to(cfg.torch_dtype)


def _calibrated(cfg, gen, blocks=1):
    nb = qw.quantwm_calib_bytes(cfg)
    calibs = torch.zeros(nb * blocks, dtype=torch.uint8, device=DEV)
    H, d, r = cfg.heads * cfg.batch, cfg.head_dim, cfg.rank
    mus = []
    for e in range(blocks):
        mu = [torch.randn(H, cfg.n_centroids, d, generator=gen, device=DEV).to(cfg.torch_dtype) for _ in range(2)]
        u = torch.linalg.qr(torch.randn(H, d, r, generator=gen, device=DEV).cpu())[0].transpose(1, 2).contiguous()
        qw.quantwm_calib_pack(cfg, *mu, torch.ones(H, d, device=DEV), u.to(DEV, cfg.torch_dtype),
                              torch.ones(H, r, device=DEV), calibs[e * nb:(e + 1) * nb])
        mus.append(mu[0])
    return calibs, nb, mus


@pytest.mark.parametrize("d,r,dtype", [(64, 4, "bf16"), (128, 6, "bf16"), (128, 32, "bf16"), (64, 13, "f32")])
def test_window_over_sparse_rows(d, r, dtype):
    """Sparse and slot-addressed PSAC rows give the same results through a window: the
    same bits where one kernel serves both, else (fp32) what the order of sums allows."""
    H, n, nq, starts = 3, 1200, 120, [0, 90, 500, 800]
    gen = torch.Generator(device=DEV).manual_seed(d + r)
    got = []
    cfgs = [qw.make_config(1, H, d, 16, 32, r, 4, n, dtype, st, coef_stage=n) for st in (0, 4)]
    calibs, cb, mus = _calibrated(cfgs[0], gen, len(starts))
    k, v, q, ka, va = (_random(cfgs[0], m, gen) for m in (n, n, nq, 50, 50))
    k[:, 5:85:2] = mus[0].view(1, H, 16, d)[:, :, 3][:, None]  # no residual: rows with scale 0 are absent
    for cfg in cfgs:
        cache = torch.zeros(qw.quantwm_cache_bytes(cfg), dtype=torch.uint8, device=DEV)
        for e, lo in enumerate(starts):
            m = (starts + [n])[e + 1] - lo
            qw.quantwm_append(cfg, calibs[e * cb:(e + 1) * cb], cache, lo, k[:, lo:lo + m].contiguous(),
                              v[:, lo:lo + m].contiguous(), m)
        for nb in (0, qw.quantwm_attend_window_workspace_bytes(cfg, n, 50, nq, 10, 100, 400)):
            ws = torch.empty(nb, dtype=torch.uint8, device=DEV) if nb else None
            out, lse = torch.full_like(q, 7.0), torch.empty((1, H, nq), device=DEV)
            qw.quantwm_attend_window(cfg, calibs, starts, cache, n, ka, va, 50, q, nq, n - 20, 10, 100, 400, out, lse, ws)
            got.append((out, lse))
    # a logit errs by (d + r + 8) 2^-24 of its terms, at most |q| |khat| / sqrt(d) with Keys decoded
    # to within their own size; a weight by that and n 2^-24, in O and in the sum; twice, for
    # either side; |vhat| is at most twice the largest Value
    size = lambda x: float(x.double().square().sum(3).max().sqrt())  # noqa: E731
    dl = (d + r + 8) * 2.0 ** -24 * size(q) * 2 * max(size(k), size(ka)) / d ** 0.5 + n * 2.0 ** -24
    for i in range(2):
        if dtype == "bf16":
            assert torch.equal(got[i][0], got[2 + i][0]) and torch.equal(got[i][1], got[2 + i][1]), i
        else:
            assert (got[i][0] - got[2 + i][0]).abs().max() <= 2 * (2 * dl + 2.0 ** -22) * 2 * float(max(v.abs().max(), va.abs().max()))
            assert (got[i][1] - got[2 + i][1]).abs().max() <= 2 * (dl + 2.0 ** -22 * float(got[i][1].abs().max()))


@pytest.mark.parametrize("nq", [1, 40, 120])
@pytest.mark.parametrize("dtype,st", [("bf16", 0), ("bf16", 1), ("f32", 0)])
def test_tiles_out_of_reach_are_not_read(dtype, st, nq):
    """Slots between the sinks' last tile and the window's first one, and past the
    cached tokens, may hold anything (bytes 0xff: NaN scales)."""
    n, n_sink, window = 1500, 70, 200
    gen = torch.Generator(device=DEV).manual_seed(3)
    cfg = qw.make_config(1, 2, 128, 16, 32, 8, 4, 1600, dtype, st)
    calibs, _, _ = _calibrated(cfg, gen)
    k, v, q = (_random(cfg, m, gen) for m in (n, n, nq))
    lo = n - nq + 1 - window  # the first Query's window
    got = []
    for fill in (0, 255):
        cache = torch.full((qw.quantwm_cache_bytes(cfg),), fill, dtype=torch.uint8, device=DEV)
        for a, b in ((0, 128), (lo // 64 * 64, n)):
            qw.quantwm_append(cfg, calibs, cache, a, k[:, a:b].contiguous(), v[:, a:b].contiguous(), b - a)
        out, lse = torch.full_like(q, 7.0), torch.empty((1, 2, nq), device=DEV)
        qw.quantwm_attend_window(cfg, calibs, [0], cache, n, None, None, 0, q, nq, n - nq, 1, n_sink, window, out, lse)
        got.append((out, lse))
    assert torch.isfinite(got[0][0].float()).all()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("nq,step", [(60, 20), (1, 20), (1, 40)])
@pytest.mark.parametrize("st", [0, 1])
def test_neighbour_epochs_of_other_magnitude(st, nq, step):
    """An epoch boundary inside a chunk, Values around 2^-100 on one side and steps near
    the largest binary16 on the other, one Query and several: neither side's keys reach
    the other's Queries as an infinity or weight."""
    H, d, kc, starts, n = 2, 128, 16, [0, 100, 200], 300
    scale = [2.0 ** -100, 2.0 ** 14, 2.0 ** -100]
    rng = np.random.default_rng(st)
    p = s64.Packed(rng, 1, H, d, kc, 32, 4, "bf16", st, [0], n)  # Keys and formats; Values and tables below
    p.tables, p.starts = [], starts
    for e, vs in enumerate(scale):
        k, v = s64.rounded(rng.standard_normal((1, 100, H, d)), "bf16"), s64.rounded(vs * rng.uniform(-1.5, 1.5, (1, 100, H, d)), "bf16")
        mu = [s64.rounded(x * rng.standard_normal((1, H, kc, d)), "bf16") for x in (1.0, vs * 2.0 ** -6)]
        u = np.stack([np.linalg.qr(rng.standard_normal((d, d)))[0][:4] for _ in range(H)])[None]
        p.tables.append((*mu, np.ones((1, H, d), np.float32), s64.rounded(u, "bf16"), np.ones((1, H, 4), np.float32)))
        oracle.append(p.ocfg, p.tables[e], p.cache, starts[e], k, v)
    q = s64.rounded(rng.standard_normal((1, nq, H, d)), "bf16")
    k, v = p.keys_values()
    # frames see windows of 100 keys, of two epochs but for step 20's first
    hi = 80 + step * (np.arange(nq) // step + 1)
    visible = (np.arange(n) < hi[:, None]) & (np.arange(n) >= hi[:, None] - 100)
    refs = [(*s64.softmax(p.logits(q, few), visible, v), s64.tolerances(q, k, n, 4, "bf16", p.residuals() if few else None))
            for few in (False, True)]
    qd = s64.dev(q, torch.bfloat16)
    out, lse = torch.full_like(qd, 7.0), torch.empty(1, H, nq, device=DEV)
    qw.quantwm_attend_window(p.cfg, p.blocks(), starts, p.on_device(), n, None, None, 0, qd, nq, 80, step, 0, 100, out, lse)
    s64.check_any(out, lse, refs)


def test_a_window_of_everything_is_attention_over_epochs():
    n, na, nq, starts = 900, 130, 300, [0, 333]
    gen = torch.Generator(device=DEV).manual_seed(5)
    cfg = qw.make_config(2, 3, 128, 32, 32, 8, 4, n, "bf16")
    calibs, cb, _ = _calibrated(cfg, gen, 2)
    k, v, q, ka, va = (_random(cfg, m, gen) for m in (n, n, nq, na, na))
    cache = torch.zeros(qw.quantwm_cache_bytes(cfg), dtype=torch.uint8, device=DEV)
    for e, (a, b) in enumerate(((0, 333), (333, n))):
        qw.quantwm_append(cfg, calibs[e * cb:(e + 1) * cb], cache, a, k[:, a:b].contiguous(), v[:, a:b].contiguous(), b - a)
    outs = [torch.full_like(q, 7.0) for _ in range(3)]
    lses = [torch.empty(2, 3, nq, device=DEV) for _ in range(3)]
    qw.quantwm_attend_epochs(cfg, calibs, starts, cache, n, ka, va, na, q, nq, 700, 30, outs[0], lses[0])
    qw.quantwm_attend_window(cfg, calibs, starts, cache, n, ka, va, na, q, nq, 700, 30, 0, n + na, outs[1], lses[1])
    qw.quantwm_attend_window(cfg, calibs, starts, cache, n, ka, va, na, q, nq, 700, 30, n + na, 0, outs[2], lses[2])
    for i in (1, 2):
        assert torch.equal(outs[i], outs[0]) and torch.equal(lses[i], lses[0])
