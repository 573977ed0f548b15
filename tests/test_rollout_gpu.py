"""The streaming calls together, as a rollout makes them: Queries and Keys of a fused
projection turned by their places, chunks appended to the packed cache, attention
through a window with the newest chunk still exact, then rollouts branching off the
history. Every output is compared with the 64-bit softmax over the cache's own decoded
contents. And the ways the calls are made: replayed from a graph, on other streams, in
the last slots of the largest cache."""
import numpy as np
import pytest
import torch

import stream64 as s64
from paper_2609_26425_amd import quantwm as qw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GRID, DIMS = (4, 5), {64: (24, 20, 20), 128: (44, 42, 42)}


def _turned(x, pos0, dims, base):
    """x [B, n, H, d] turned by the places pos0 + i of the grid, adjacent pairs, in 64 bits."""
    n = x.shape[1]
    at = pos0 + np.arange(n)
    place = np.stack([at // 20, at // 5 % 4, at % 5], 1).astype(np.float64)
    ang = np.concatenate([place[:, a:a + 1] * base ** (-np.arange(0, D, 2) / D) for a, D in enumerate(dims)], 1)
    c, s = np.cos(ang)[None, :, None], np.sin(ang)[None, :, None]
    out = np.empty_like(x)
    out[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    out[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    return out


@pytest.mark.parametrize("dtype,d,st", [("bf16", 128, 0), ("bf16", 64, 1), ("f32", 64, 0)])
def test_a_rollout_and_its_branches(dtype, d, st):
    H, F, chunk, n_chunks, window, n_sink = 2, 20, 60, 6, 140, 20
    rng = np.random.default_rng(d + st)
    p = s64.Packed(rng, 1, H, d, 16, 32, 8, dtype, st, [0, 180], chunk * n_chunks)  # two epochs' tables
    p.cache[:] = 0
    dt, blocks, cb = p.cfg.torch_dtype, p.blocks(), qw.quantwm_calib_bytes(p.cfg)
    cache = torch.zeros(qw.quantwm_cache_bytes(p.cfg), dtype=torch.uint8, device=DEV)
    axes = qw.rotary_axes(p.cfg, DIMS[d], *GRID)
    q, k = (torch.empty(1, chunk, H, d, dtype=dt, device=DEV) for _ in range(2))
    for c in range(n_chunks):
        x = s64.rounded(rng.standard_normal((1, chunk, 3, H, d)), dtype)
        qkv = s64.dev(x, dt)
        qw.quantwm_rotary(p.cfg, axes, qkv[:, :, 0], qkv[:, :, 1], chunk, q, k, pos0=c * chunk)
        v = qkv[:, :, 2].contiguous()
        for got, i in ((q, 0), (k, 1)):  # half a step of the type, and the fp32 turn
            ref = _turned(x[:, :, i].astype(np.float64), c * chunk, DIMS[d], 1e4)
            assert (np.abs(got.double().cpu().numpy() - ref) <= (2.0 ** -8 if dtype == "bf16" else 0) * np.abs(ref) + 2.0 ** -20 * 8).all()
        done = c * chunk
        starts = p.starts[:1 if done <= 180 else 2]
        out, lse = torch.full_like(q, 7.0), torch.empty(1, H, chunk, device=DEV)
        qw.quantwm_attend_window(p.cfg, blocks, starts, cache, done, k, v, chunk, q, chunk, done, F, n_sink, window, out, lse)
        # against the cache as it is
        p.cache[:] = cache.cpu().numpy()
        n = done + chunk
        hi = done + (np.arange(chunk) // F + 1) * F
        j = np.arange(n)
        visible = (j < hi[:, None]) & ((j < n_sink) | (j >= hi[:, None] - window))
        qn, kn, vn = (t.float().cpu().numpy() for t in (q, k, v))
        full, (p.n, p.starts) = (p.n, p.starts), (done, starts)
        pk, pv = p.keys_values()
        kk, vv = (np.concatenate([a[:, :, :done], b.transpose(0, 2, 1, 3)], 2) for a, b in ((pk, kn), (pv, vn)))
        refs = []
        for few in s64.forms(dtype):
            lg = np.concatenate([p.logits(qn, few), s64.exact_logits(qn, kn)], 3)
            refs.append((*s64.softmax(lg, visible, vv), s64.tolerances(qn, kk, n, 8, dtype, p.residuals() if few else None)))
        p.n, p.starts = full
        s64.check_any(out, lse, refs)
        e = int(done >= 180)
        qw.quantwm_append(p.cfg, blocks[e * cb:(e + 1) * cb], cache, done, k, v, chunk)
    # three rollouts of one frame off this history, their first tokens packed, the last exact
    p.cache[:] = cache.cpu().numpy()
    B, n_pk, n_act = 3, 12, 8
    own = s64.Packed(rng, B, H, d, 16, 32, 8, dtype, st, [0], n_pk)
    qn, ka, va = (s64.rounded(rng.standard_normal((B, n_act, H, d)), dtype) for _ in range(3))
    total = chunk * n_chunks
    nb = qw.quantwm_attend_shared_workspace_bytes(p.cfg, total, own.cfg, n_pk, n_act, n_act)
    ws, qd = torch.empty(nb, dtype=torch.uint8, device=DEV), s64.dev(qn, dt)
    out, lse = torch.full_like(qd, 7.0), torch.empty(B, H, n_act, device=DEV)
    qw.quantwm_attend_shared(p.cfg, blocks, p.starts, cache, total, own.cfg, own.blocks(), own.on_device(), n_pk,
                             s64.dev(ka, dt), s64.dev(va, dt), n_act, qd, n_act, total + n_pk, F, out, lse, ws)
    pk, pv = p.keys_values()
    k, v = own.keys_values()
    kk, vv = (np.concatenate([np.repeat(a, B, 0), b, x.transpose(0, 2, 1, 3)], 2) for a, b, x in ((pk, k, ka), (pv, v, va)))
    n = kk.shape[2]
    visible = np.arange(n) < (total + n_pk + (np.arange(n_act) // F + 1) * F)[:, None]
    flat, refs = qn.reshape(1, B * n_act, H, d), []
    for fp in s64.forms(dtype):
        for fo in s64.forms(dtype):
            lg = np.concatenate([p.logits(flat, fp).reshape(H, B, n_act, total).transpose(1, 0, 2, 3), own.logits(qn, fo),
                                 s64.exact_logits(qn, ka)], 3)
            res = np.concatenate([np.repeat(p.residuals(), B, 0), own.residuals()], 2) if fp or fo else None
            refs.append((*s64.softmax(lg, visible, vv), s64.tolerances(qn, kk, 2 * n + 64, 8, dtype, res)))
    s64.check_any(out, lse, refs)


class _Calls:
    """One of each call on inputs of its own, with its buffers."""

    def __init__(self, dtype, nq, seed):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.nq, self.n, self.na, self.B, H, d = nq, 2000, 40, 3, 2, 128
        R = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(self.cfg.torch_dtype)  # noqa: E731
        self.cfg = qw.make_config(1, H, d, 32, 32, 8, 4, self.n, dtype)
        self.own = qw.make_config(self.B, H, d, 32, 32, 8, 4, 64, dtype)
        self.blocks = []
        for cfg in (self.cfg, self.own):
            bh = cfg.batch * H
            u = torch.linalg.qr(torch.randn(bh, d, 8, generator=gen, device=DEV).cpu())[0].transpose(1, 2).contiguous()
            blk = torch.zeros(qw.quantwm_calib_bytes(cfg), dtype=torch.uint8, device=DEV)
            qw.quantwm_calib_pack(cfg, R(bh, 32, d), R(bh, 32, d), torch.ones(bh, d, device=DEV),
                                  u.to(DEV, cfg.torch_dtype), torch.ones(bh, 8, device=DEV), blk)
            self.blocks.append(blk)
        self.caches = [torch.zeros(qw.quantwm_cache_bytes(c), dtype=torch.uint8, device=DEV) for c in (self.cfg, self.own)]
        for cfg, blk, cache, n in zip((self.cfg, self.own), self.blocks, self.caches, (self.n, 64)):
            qw.quantwm_append(cfg, blk, cache, 0, R(cfg.batch, n, H, d), R(cfg.batch, n, H, d), n)
        self.x, self.k, self.v = R(1, nq, H, d), R(1, self.na, H, d), R(1, self.na, H, d)
        self.y, self.ky, self.vy = R(self.B, nq, H, d), R(self.B, self.na, H, d), R(self.B, self.na, H, d)
        self.axes = qw.rotary_axes(self.cfg, DIMS[d], *GRID)
        self.q, self.out = torch.empty_like(self.x), torch.empty_like(self.x)
        self.lse, self.shared = torch.empty(1, H, nq, device=DEV), torch.empty_like(self.y)
        new = lambda nb: torch.empty(max(256, nb), dtype=torch.uint8, device=DEV)  # noqa: E731
        self.ws = new(qw.quantwm_attend_window_workspace_bytes(self.cfg, self.n, self.na, nq, 1, 30, 1500))
        self.ws2 = new(qw.quantwm_attend_shared_workspace_bytes(self.cfg, self.n, self.own, 64, self.na, nq))

    def run(self, stream=None):
        end = self.n + self.na
        qw.quantwm_rotary(self.cfg, self.axes, self.x, None, self.nq, self.q, pos0=777, stream=stream)
        qw.quantwm_attend_window(self.cfg, self.blocks[0], [0], self.caches[0], self.n, self.k, self.v, self.na, self.q,
                                 self.nq, end - self.nq, 1, 30, 1500, self.out, self.lse, self.ws, stream=stream)
        qw.quantwm_attend_shared(self.cfg, self.blocks[0], [0], self.caches[0], self.n, self.own, self.blocks[1],
                                 self.caches[1], 64, self.ky, self.vy, self.na, self.y, self.nq,
                                 self.n + 64 + max(0, self.na - self.nq), 1, self.shared, None, self.ws2, stream=stream)

    def results(self):
        return [t.clone() for t in (self.q, self.out, self.lse, self.shared)]


def _same(a, b):
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype,nq", [("bf16", 1), ("bf16", 5), ("bf16", 300), ("f32", 33)])
def test_replayed_from_a_graph(dtype, nq):
    c = _Calls(dtype, nq, nq)
    c.run()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.run()
    for i in range(4):  # new inputs in place, with eager work in between
        c.x.mul_(1.0 + 0.25 * i)
        c.y.add_(0.125 * i)
        graph.replay()
        torch.cuda.synchronize()
        got = c.results()
        for t in (c.q, c.out, c.lse, c.shared, c.ws, c.ws2):
            t.fill_(3)
        c.run()
        torch.cuda.synchronize()
        _same(got, c.results())


def test_on_other_streams_and_two_at_once():
    cs = [_Calls("bf16", nq, nq) for nq in (3, 290)]
    want = []
    for c in cs:
        c.run()
        want.append(c.results())
        for t in (c.q, c.out, c.lse, c.shared):
            t.fill_(7)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(3):
        for c, s in zip(cs, streams):  # as a Stream, and as the current one
            c.run(stream=s)
            with torch.cuda.stream(s):
                c.run()
    torch.cuda.synchronize()
    for c, w in zip(cs, want):
        _same(c.results(), w)


@pytest.mark.parametrize("nq", [1, 100])
def test_the_last_slots_of_the_largest_cache(nq):
    """2^26 slots (2 GiB of codes a side): a window at their end gives the bits that it gives
    in a small cache, which an offset past 32 bits would not."""
    H, d, r, n_sink, window = 1, 128, 32, 100, 1000
    gen = torch.Generator(device=DEV).manual_seed(9)
    R = lambda *s: torch.randn(*s, generator=gen, device=DEV).bfloat16()  # noqa: E731
    k, v, q = R(1, 1280, H, d), R(1, 1280, H, d), R(1, nq, H, d)
    mu, u = [R(H, 256, d) for _ in range(2)], torch.linalg.qr(torch.randn(H, d, r, generator=gen, device=DEV).cpu())[0]
    got = []
    for n in (8192, 1 << 26):
        cfg = qw.make_config(1, H, d, 256, 16, r, 4, n, "bf16")
        blk = torch.zeros(qw.quantwm_calib_bytes(cfg), dtype=torch.uint8, device=DEV)
        qw.quantwm_calib_pack(cfg, *mu, torch.ones(H, d, device=DEV), u.transpose(1, 2).contiguous().to(DEV).bfloat16(),
                              torch.ones(H, r, device=DEV), blk)
        cache = torch.zeros(qw.quantwm_cache_bytes(cfg), dtype=torch.uint8, device=DEV)
        qw.quantwm_append(cfg, blk, cache, 0, k[:, :128].contiguous(), v[:, :128].contiguous(), 128)
        qw.quantwm_append(cfg, blk, cache, n - 1152, k[:, 128:].contiguous(), v[:, 128:].contiguous(), 1152)
        nb = qw.quantwm_attend_window_workspace_bytes(cfg, n, 0, nq, 1, n_sink, window)
        for ws in (None, torch.empty(max(256, nb), dtype=torch.uint8, device=DEV)):
            out, lse = torch.full_like(q, 7.0), torch.empty(1, H, nq, device=DEV)
            qw.quantwm_attend_window(cfg, blk, [0], cache, n, None, None, 0, q, nq, n - nq, 1, n_sink, window, out, lse, ws)
            got.append((out, lse))
        torch.cuda.synchronize()
        del cache
    for i in range(2):
        _same(got[i], got[2 + i])
    assert torch.isfinite(got[0][0].float()).all() and float(got[0][0].float().abs().max()) > 0
