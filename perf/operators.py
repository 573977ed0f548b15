"""Rotary positions, windowed attention and shared-history attention of a streaming
video world model, in plain form and through the package's entry points.

A rollout turns its chunk's Queries and Keys by their places in the video (frame,
row, column), appends them to the packed 2-bit cache and attends through a window
of the last frames beside a few first tokens that stay visible. A planner branches
several rollouts off one packed history. The listed cases take these calls at the
shapes of the repository's workloads (12, 30 and 40 heads, the small fp32 one);
draw() takes them over the same ranges.

Inputs are synthetic, with the statistics of normalised Queries and Keys: Keys
around centroids with channel scales and a few larger channels, Queries with a
dominant subspace. Packed caches are quantised here, in torch, by the rules of
the packed format (include/quantwm.h), so that they depend on the seed alone.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"

# The workloads' shapes: heads, head_dim, centroids, group, PSAC rank, and the
# rows and columns of a frame's tokens.
_MG2 = dict(batch=1, heads=12, d=128, kc=64, g=32, r=8, gh=22, gw=40, dtype="bf16", storage=0)
_LING = dict(batch=1, heads=40, d=128, kc=128, g=32, r=16, gh=30, gw=52, dtype="bf16", storage=0)
_BATCH = dict(batch=4, heads=30, d=128, kc=256, g=64, r=32, gh=26, gw=40, dtype="bf16", storage=0)
_TINY = dict(batch=1, heads=2, d=64, kc=16, g=32, r=4, gh=5, gw=10, dtype="f32", storage=0)


def listed():
    rot = dict(kind="rotary", pairs="adjacent", explicit=False, inverse=False, fused=False, base=10000.0)
    win = dict(kind="window", epochs=1, n_act=0)
    return [
        # one token of a 12-head model (an action or register token): latency
        dict(_MG2 | rot, name="rotary-token", n=1, pos0=41_360),
        # the 3-frame chunk of the 40-head model, Queries and Keys, late in a rollout
        dict(_LING | rot, name="rotary-chunk", n=4680, pos0=1_170_000),
        # gradient of four rollouts' frames in a fused projection [B, n, 3, H, d],
        # tokens gathered in another order (explicit positions), halves paired
        dict(_BATCH | rot, name="rotary-gradient", n=1037, pos0=0, pairs="halves", explicit=True, inverse=True, fused=True),
        # the small fp32 path, an odd number of tokens
        dict(_TINY | rot, name="rotary-f32", n=257, pos0=900, explicit=True),
        # one Query over a long cache: causal by tokens, 9 frames of window
        dict(_LING | win, name="window-token", n_cache=32_760, n_q=1, q_start=32_759, frame=1, n_sink=1560, window=14_040),
        # one frame of Queries of the 12-head model, 5 frames of window
        dict(_MG2 | win, name="window-frame", n_cache=13_200, n_q=880, q_start=12_320, frame=880, n_sink=880, window=4400),
        # the 40-head chunk, still exact, over a recalibrated history with 8-bit
        # group scales: the first frame and the last 9
        dict(_LING | win, name="window-chunk", n_cache=28_080, n_act=4680, n_q=4680, q_start=28_080, frame=1560,
             n_sink=1560, window=14_040, epochs=6, storage=1),
        # the small fp32 path: causal by tokens, bounds inside tiles
        dict(_TINY | win, name="window-f32", n_cache=1200, n_act=57, n_q=257, q_start=1000, frame=1, n_sink=5, window=300),
        # sixteen candidate actions of a planner, one token each, off one history
        dict(_BATCH, kind="shared", name="shared-tokens", batch=16, n_prefix=24_960, n_cache=130, n_act=1, n_q=1,
             frame=1, prefix_epochs=1),
        # four rollouts one frame into the future, the second frame still exact
        dict(_BATCH, kind="shared", name="shared-frames", n_prefix=24_960, n_cache=1040, n_act=1040, n_q=1040,
             frame=1040, prefix_epochs=4),
        # the small fp32 path: three rollouts of odd lengths
        dict(_TINY, kind="shared", name="shared-f32", batch=3, n_prefix=777, n_cache=70, n_act=33, n_q=33, frame=1,
             prefix_epochs=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "window", "window", "shared"])
    f32 = rng.random() < 0.25
    d = rng.choice([64, 128, 128])
    c = dict(kind=kind, batch=rng.choice([1, 1, 2, 4]), heads=_log(rng, 2, 8) if f32 else _log(rng, 4, 40), d=d,
             kc=_log(rng, 16, 256), g=rng.choice([16, 32, 64]), r=rng.choice([0, 4, 8, 12, 16, 24, 32]),
             gh=_log(rng, 4, 30), gw=_log(rng, 5, 52), dtype="f32" if f32 else "bf16", storage=0)
    if kind == "rotary":
        c.update(n=_log(rng, 1, 4680), pos0=_log(rng, 1, 2_000_000), pairs=rng.choice(["adjacent", "halves"]),
                 explicit=rng.random() < 0.5, inverse=rng.random() < 0.3, fused=rng.random() < 0.3, base=rng.choice([1e4, 1e6]))
        c["n"] = max(1, min(c["n"], 187_000 // (c["batch"] * c["heads"])))
        return c
    c["storage"] = rng.choice([0, 0, 1])
    frame = c["gh"] * c["gw"]
    c["frame"] = rng.choice([1, frame, frame])
    c["n_q"] = rng.choice([rng.randint(1, 8), frame, _log(rng, 16, 1024 if f32 else 4680)])
    hist = _log(rng, 200, 3000 if f32 else 30_000)
    if kind == "window":
        c["n_act"] = rng.choice([0, 0, c["n_q"], rng.randint(1, 200)])
        c["n_cache"] = hist
        c["q_start"] = max(0, hist + c["n_act"] - c["n_q"])
        c["n_sink"] = rng.choice([0, rng.randint(1, 64), frame])
        c["window"] = max(c["frame"], _log(rng, 64, 15_000))  # a frame sees itself
        c["epochs"] = rng.randint(1, max(1, min(7, hist // 100)))
    else:
        c["batch"] = rng.choice([2, 3, 4, 8, 16])
        c.update(n_prefix=hist, n_cache=rng.choice([0, rng.randint(1, 300), frame]), n_act=rng.choice([0, c["n_q"]]),
                 prefix_epochs=rng.randint(1, max(1, min(7, hist // 100))))
        c["n_cache"] = c["n_cache"] or (0 if c["n_act"] else 64)
    most = 2e11 if f32 else 1.3e12
    while c["n_q"] > 1 and (work(c)["flops"] > most or c["batch"] * c["heads"] * c["n_q"] > 187_200):
        old, c["n_q"] = c["n_q"], max(1, c["n_q"] // 2)
        if c["n_act"] == old:
            c["n_act"] = c["n_q"]
        if kind == "window":
            c["q_start"] = max(0, c["n_cache"] + c["n_act"] - c["n_q"])
    return c


# ------------------------------------------------------------------ inputs


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _rows(x):
    """[B, n, H, d] -> [B*H, n, d]."""
    b, n, h, d = x.shape
    return x.transpose(1, 2).reshape(b * h, n, d)


def _sections(case, bh, capacity):
    """Byte offsets and bytes per token of the packed cache's sections, the slots
    of a head and the bytes of the cache."""
    d, r, i8, ng = case["d"], case["r"], case["storage"] & 1, case["d"] // case["g"]
    slots = (capacity + 63) // 64 * 64
    side = [("codes", d // 4), ("ids", 1), ("zp", (ng + 3) // 4), ("scale", ng if i8 else 2 * ng)]
    names = [("k_" + n, p) for n, p in side] + [("k_coef", r), ("k_cscale", 2 if r else 0)]
    names += [("v_" + n, p) for n, p in side] + [("k_sigma", 2 if i8 else 0), ("v_sigma", 2 if i8 else 0)]
    out, at = {}, 0
    for n, p in names:
        out[n] = (at, p)
        at = (at + bh * slots * p + 255) // 256 * 256
    return out, slots, at


def _bits2(x):
    """2-bit fields [bh, n, f] to bytes [bh, n, ceil(f / 4)]."""
    h, n, f = x.shape
    if f % 4:
        x = torch.cat([x, x.new_zeros(h, n, 4 - f % 4)], 2)
    x = x.view(h, n, x.shape[2] // 4, 4)
    return x[..., 0] | (x[..., 1] << 2) | (x[..., 2] << 4) | (x[..., 3] << 6)


class _Source:
    """The seeded streams of one case: channel statistics per head, then Keys,
    Values and Queries."""

    def __init__(self, case, seed):
        self.case, self.d = case, case["d"]
        self.gen = torch.Generator(device=DEV).manual_seed(9_176_263 * seed + 29)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen, device=DEV)

    def heads(self, bh):
        sigma = (0.4 * self.normal(bh, self.d)).exp()
        sigma[:, :4] *= 3.0
        order = torch.rand(bh, self.d, generator=self.gen, device=DEV).argsort(1)
        sigma = sigma.gather(1, order)
        self.sigma = sigma / sigma.square().mean(1, keepdim=True).sqrt()
        rank = max(4, self.case["r"])
        self.basis = torch.linalg.qr(self.normal(bh, self.d, rank).cpu())[0].to(DEV).transpose(1, 2).contiguous()

    def bnhd(self, x, batch):  # [BH, n, d] -> [B, n, H, d]
        return x.to(_dt(self.case)).view(batch, -1, x.shape[1], self.d).transpose(1, 2).contiguous()

    def queries(self, batch, n):
        bh = self.basis.shape[0]
        bh_q = batch * self.case["heads"]
        basis = self.basis.repeat(bh_q // bh, 1, 1)
        x = self.normal(bh_q, n, self.d) + 1.5 * torch.bmm(self.normal(bh_q, n, basis.shape[1]), basis)
        return self.bnhd(x, batch)

    def exact_rows(self, batch, n):
        """Keys and Values of an exact chunk, [B, n, H, d]."""
        bh_k = batch * self.case["heads"]
        sig = self.sigma.repeat(bh_k // self.sigma.shape[0], 1)
        return self.bnhd(self.normal(bh_k, n, self.d) * sig[:, None, :], batch), self.bnhd(self.normal(bh_k, n, self.d), batch)

    def tables(self, bh):
        """Method-level tables of one calibration block."""
        c = self.case
        sig = self.sigma.repeat(bh // self.sigma.shape[0], 1)
        basis = self.basis.repeat(bh // self.basis.shape[0], 1, 1)
        mu_k = (0.85 * self.normal(bh, c["kc"], self.d) * sig[:, None, :]).to(_dt(c))
        mu_v = (0.6 * self.normal(bh, c["kc"], self.d)).to(_dt(c))
        u = basis[:, :c["r"]].to(_dt(c)).contiguous() if c["r"] else None
        return dict(mu_k=mu_k, mu_v=mu_v, u=u)

    def packed(self, bh, capacity, starts, n, tables):
        """A packed cache of n tokens per head, quantised with tables[e] from
        starts[e] on: centroid, INT2 residual with a zero-point per group, INT8
        coefficients of the remaining Key error."""
        c, d, g = self.case, self.d, self.case["g"]
        sec, slots, total = _sections(c, bh, max(1, capacity))
        cache = torch.zeros(total, dtype=torch.uint8, device=DEV)

        def put(name, lo, x):
            at, per = sec[name]
            cache[at:at + bh * slots * per].view(bh, slots, per)[:, lo:lo + x.shape[1]] = x

        for t, lo, hi in zip(tables, starts, starts[1:] + [n]):
            m = hi - lo
            if m == 0:
                continue
            for side, mu, spread in (("k_", t["mu_k"], 0.5), ("v_", t["mu_v"], 0.8)):
                ids = torch.randint(c["kc"], (bh, m), generator=self.gen, device=DEV)
                e = spread * self.normal(bh, m, d)
                if side == "k_":
                    e *= self.sigma.repeat(bh // self.sigma.shape[0], 1)[:, None, :]
                e = e.view(bh, m, d // g, g)
                low, high = e.amin(3).clamp(max=0.0), e.amax(3).clamp(min=0.0)
                step = (high - low) / 3.0
                if c["storage"] & 1:
                    sig = (step.amax(2, keepdim=True) / 255.0).half().float()
                    code = (step / sig).round().clamp(1, 255)
                    put(side + "scale", lo, code.to(torch.uint8))
                    put(side + "sigma", lo, sig.half().view(torch.uint8))
                    step = sig * code
                else:
                    step = step.half().float()
                    put(side + "scale", lo, step.half().view(torch.uint8))
                zp = (-low / step).round().clamp(0, 3)
                q = ((e / step[..., None]).round() + zp[..., None]).clamp(0, 3)
                put(side + "codes", lo, _bits2(q.view(bh, m, d).to(torch.uint8)))
                put(side + "zp", lo, _bits2(zp.to(torch.uint8)))
                put(side + "ids", lo, ids.to(torch.uint8)[:, :, None])
                if side == "k_" and c["r"]:
                    err = (e - step[..., None] * (q - zp[..., None])).view(bh, m, d)
                    cf = torch.bmm(err, t["u"].float().transpose(1, 2).contiguous())
                    cs = (cf.abs().amax(2, keepdim=True) / 127.0).half()
                    put("k_coef", lo, (cf / cs.float()).round().clamp(-127, 127).to(torch.int8).view(torch.uint8))
                    put("k_cscale", lo, cs.view(torch.uint8))
        return cache


def _starts(n, epochs):
    return [e * n // epochs for e in range(epochs)]


def _freq(case):
    """Angle per unit of position of every pair, and the pair's axis: base^(-2 i / D)
    on the D channels of each axis (height and width a sixth of the pairs' two each)."""
    d, side = case["d"], 2 * (case["d"] // 6)
    dims = (d - 2 * side, side, side)
    freq = [case["base"] ** (-2.0 * i / D) for D in dims for i in range(D // 2)]
    return dims, freq, [a for a, D in enumerate(dims) for _ in range(D // 2)]


def _inputs(case, seed):
    """Everything the operators read, the same for both forms."""
    c, s = case, _Source(case, seed)
    B, H, d = c["batch"], c["heads"], c["d"]
    if c["kind"] == "rotary":
        n = c["n"]
        if c["fused"]:
            qkv = s.normal(B, n, 3, H, d).to(_dt(c))
            q, k = qkv[:, :, 0], qkv[:, :, 1]
        else:
            q, k = s.normal(B, n, H, d).to(_dt(c)), s.normal(B, n, H, d).to(_dt(c))
        pos = None
        if c["explicit"]:
            at = c["pos0"] + torch.rand(B, n, generator=s.gen, device=DEV).argsort(1)
            area = c["gh"] * c["gw"]
            pos = torch.stack([at // area, at // c["gw"] % c["gh"], at % c["gw"]], 2).to(torch.int32)
        return dict(case=c, q=q, k=k, pos=pos)
    if c["kind"] == "window":
        s.heads(B * H)
        starts = _starts(c["n_cache"], c["epochs"])
        tables = [s.tables(B * H) for _ in starts]
        cache = s.packed(B * H, c["n_cache"], starts, c["n_cache"], tables)
        ka, va = s.exact_rows(B, c["n_act"]) if c["n_act"] else (None, None)
        return dict(case=c, starts=starts, tables=tables, cache=cache, ka=ka, va=va, q=s.queries(B, c["n_q"]))
    s.heads(H)
    starts = _starts(c["n_prefix"], c["prefix_epochs"])
    ptables = [s.tables(H) for _ in starts]
    prefix = s.packed(H, c["n_prefix"], starts, c["n_prefix"], ptables)
    tables = s.tables(B * H)
    cache = s.packed(B * H, c["n_cache"], [0], c["n_cache"], [tables])
    ka, va = s.exact_rows(B, c["n_act"]) if c["n_act"] else (None, None)
    return dict(case=c, starts=starts, ptables=ptables, prefix=prefix, tables=[tables], cache=cache, ka=ka, va=va,
                q=s.queries(B, c["n_q"]))


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _handles(st)
    return st


def _shared_start(c):
    """Position of the first Query: the last n_q of all the positions, behind the prefix."""
    return c["n_prefix"] + max(0, c["n_cache"] + c["n_act"] - c["n_q"])


def _handles(st):
    """What a user's program keeps beside the inputs: the configuration, the
    calibration blocks on the device, workspaces and output buffers."""
    from paper_2609_26425_amd import quantwm as qw
    c = st["case"]
    st["qw"] = qw

    def config(batch, capacity):
        return qw.make_config(batch, c["heads"], c["d"], c["kc"], c["g"], c["r"], 4, max(1, capacity), c["dtype"],
                              storage=c["storage"])

    def blocks(cfg, tables):
        nb = qw.quantwm_calib_bytes(cfg)
        out = torch.zeros(nb * len(tables), dtype=torch.uint8, device=DEV)
        w = torch.ones(cfg.batch * cfg.heads, c["d"], device=DEV)
        for e, t in enumerate(tables):
            qw.quantwm_calib_pack(cfg, t["mu_k"], t["mu_v"], w, t["u"], None, out[e * nb:(e + 1) * nb])
        return out

    def scratch(nb):
        return torch.empty(nb, dtype=torch.uint8, device=DEV) if nb else None

    if c["kind"] == "rotary":
        dims, _, _ = _freq(c)
        st["cfg"] = config(c["batch"], 1)
        pairs = qw.ROTARY_ADJACENT if c["pairs"] == "adjacent" else qw.ROTARY_HALVES
        st["axes"] = qw.rotary_axes(st["cfg"], dims, c["gh"], c["gw"], base=c["base"], pairs=pairs)
        st["qo"], st["ko"] = (torch.empty(st["q"].shape, dtype=_dt(c), device=DEV) for _ in range(2))
        return
    st["out"] = torch.empty_like(st["q"])
    # fp32 callers take the log-sum-exp too
    st["lse"] = torch.empty(c["batch"], c["heads"], c["n_q"], device=DEV) if c["dtype"] == "f32" else None
    st["cfg"] = config(c["batch"], c["n_cache"])
    st["calib"] = blocks(st["cfg"], st["tables"])
    if c["kind"] == "window":
        st["ws"] = scratch(qw.quantwm_attend_window_workspace_bytes(st["cfg"], c["n_cache"], c["n_act"], c["n_q"],
                                                                    c["frame"], c["n_sink"], c["window"]))
        return
    st["pcfg"] = config(1, c["n_prefix"])
    st["pcalib"] = blocks(st["pcfg"], st["ptables"])
    st["ws"] = scratch(qw.quantwm_attend_shared_workspace_bytes(st["pcfg"], c["n_prefix"], st["cfg"], c["n_cache"],
                                                                c["n_act"], c["n_q"]))


def run(st):
    return _own(st) if own else _plain(st)


def _own(st):
    c, qw = st["case"], st["qw"]
    if c["kind"] == "rotary":
        qw.quantwm_rotary(st["cfg"], st["axes"], st["q"], st["k"], c["n"], st["qo"], st["ko"], pos0=c["pos0"],
                          pos=st["pos"], inverse=c["inverse"])
        return dict(q=st["qo"], k=st["ko"])
    if c["kind"] == "window":
        qw.quantwm_attend_window(st["cfg"], st["calib"], st["starts"], st["cache"], c["n_cache"], st["ka"], st["va"],
                                 c["n_act"], st["q"], c["n_q"], c["q_start"], c["frame"], c["n_sink"], c["window"],
                                 st["out"], st["lse"], st["ws"])
    else:
        qw.quantwm_attend_shared(st["pcfg"], st["pcalib"], st["starts"], st["prefix"], c["n_prefix"], st["cfg"],
                                 st["calib"], st["cache"], c["n_cache"], st["ka"], st["va"], c["n_act"], st["q"],
                                 c["n_q"], _shared_start(c), c["frame"], st["out"], st["lse"], st["ws"])
    return dict(out=st["out"]) if st["lse"] is None else dict(out=st["out"], lse=st["lse"])


# -------------------------------------------------------------- plain forms


def _plain(st):
    c = st["case"]
    if c["kind"] == "rotary":
        return _plain_rotary(st)
    out, lse = _plain_window(st) if c["kind"] == "window" else _plain_shared(st)
    out = out.view(c["batch"], c["heads"], c["n_q"], c["d"]).transpose(1, 2).contiguous().to(_dt(c))
    return dict(out=out) if c["dtype"] == "bf16" else dict(out=out, lse=lse.view(c["batch"], c["heads"], c["n_q"]))


def _plain_rotary(st):
    c = st["case"]
    _, freq, axis = _freq(c)
    if st["pos"] is None:
        at = c["pos0"] + torch.arange(c["n"], device=DEV)[None]
        area = c["gh"] * c["gw"]
        pos = torch.stack([at // area, at // c["gw"] % c["gh"], at % c["gw"]], 2)
    else:
        pos = st["pos"]
    # far positions: angles in 64 bits
    ang = pos.double()[:, :, axis] * torch.tensor(freq, dtype=torch.float64, device=DEV)
    cos, sin = ang.cos().float()[:, :, None, :], ang.sin().float()[:, :, None, :]
    if c["inverse"]:
        sin = -sin

    def turn(x):
        x = x.float()
        half = c["d"] // 2
        if c["pairs"] == "adjacent":
            a, b = x[..., 0::2], x[..., 1::2]
            return torch.stack([a * cos - b * sin, a * sin + b * cos], 4).flatten(3).to(_dt(c))
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], 3).to(_dt(c))

    return dict(q=turn(st["q"]), k=turn(st["k"]))


def _field(case, cache, bh, capacity, name):
    sec, slots, _ = _sections(case, bh, max(1, capacity))
    at, per = sec[name]
    return cache[at:at + bh * slots * per].view(bh, slots, per)


def _two(x, f):
    """The first f 2-bit fields of bytes [bh, n, m] as float32."""
    sh = torch.tensor([0, 2, 4, 6], device=DEV, dtype=torch.uint8)
    return ((x[..., None] >> sh) & 3).flatten(2)[:, :, :f].float()


def _dequant(case, cache, bh, capacity, starts, at, tables):
    """Keys (with their correction, U_r c added) and Values of the slots `at` of a
    packed cache, [bh, n, d] float32."""
    d, g, r = case["d"], case["g"], case["r"]
    if not at.numel():
        return [torch.empty(bh, 0, d, device=DEV) for _ in range(2)]
    epoch = torch.bucketize(at, torch.tensor(starts, device=DEV), right=True) - 1
    head = torch.arange(bh, device=DEV)[:, None]
    got = []
    for side in ("k_", "v_"):
        get = lambda name: _field(case, cache, bh, capacity, name)[:, at].contiguous()  # noqa: E731
        scale = get(side + "scale")
        if case["storage"] & 1:
            scale = scale.float() * get(side + "sigma").view(torch.float16).float()
        else:
            scale = scale.view(torch.float16).float()
        q, zp = _two(get(side + "codes"), d).view(bh, -1, d // g, g), _two(get(side + "zp"), d // g)
        mu = torch.stack([t["mu_" + side[0]] for t in tables])
        x = mu[epoch[None, :], head, get(side + "ids")[:, :, 0].long()].float()
        got.append(x + (scale[..., None] * (q - zp[..., None])).view(bh, -1, d))
    if r:
        coef = get("k_coef").view(torch.int8).float() * get("k_cscale").view(torch.float16).float()
        place = torch.nn.functional.one_hot(epoch, len(tables)).float()  # a row's ranks in its epoch's place
        coef = (place[None, :, :, None] * coef[:, :, None, :]).flatten(2)
        got[0] += torch.bmm(coef, torch.cat([t["u"] for t in tables], 1).float())
    return got


def _softmax(logits, visible, v):
    """softmax over the visible keys times v, and the log-sum-exp; a row without a
    visible key gives zeros and -inf."""
    logits = logits.masked_fill_(~visible, -math.inf)
    top = logits.amax(2, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = logits.sub_(top).exp_()
    total = p.sum(2, keepdim=True)
    out = torch.bmm(p, v) / torch.where(total > 0, total, torch.ones_like(total))
    return out, (top + total.log())[:, :, 0]


def _plain_window(st):
    c = st["case"]
    bh, nk = c["batch"] * c["heads"], c["n_cache"] + c["n_act"]
    hi = c["q_start"] + (torch.arange(c["n_q"], device=DEV) // c["frame"] + 1) * c["frame"]
    # the keys that some Query sees
    low = min(nk, max(c["n_sink"], c["q_start"] + c["frame"] - c["window"]))
    high = min(nk, c["q_start"] + ((c["n_q"] - 1) // c["frame"] + 1) * c["frame"])
    at = torch.cat([torch.arange(min(c["n_sink"], high), device=DEV), torch.arange(low, max(low, high), device=DEV)])
    packed, exact_ = at[at < c["n_cache"]], at[at >= c["n_cache"]] - c["n_cache"]
    k, v = _dequant(c, st["cache"], bh, c["n_cache"], st["starts"], packed, st["tables"])
    if c["n_act"]:
        k = torch.cat([k, _rows(st["ka"])[:, exact_].float()], 1)
        v = torch.cat([v, _rows(st["va"])[:, exact_].float()], 1)
    q = _rows(st["q"]).float() / math.sqrt(c["d"])
    visible = (at < hi[:, None]) & ((at < c["n_sink"]) | (at >= hi[:, None] - c["window"]))
    return _softmax(torch.bmm(q, k.transpose(1, 2).contiguous()), visible, v)


def _plain_shared(st):
    c = st["case"]
    B, H, nq, d = c["batch"], c["heads"], c["n_q"], c["d"]
    n_own = c["n_cache"] + c["n_act"]
    pk, pv = _dequant(c, st["prefix"], H, c["n_prefix"], st["starts"], torch.arange(c["n_prefix"], device=DEV), st["ptables"])
    k, v = _dequant(c, st["cache"], B * H, c["n_cache"], [0], torch.arange(c["n_cache"], device=DEV), st["tables"])
    if c["n_act"]:
        k, v = torch.cat([k, _rows(st["ka"]).float()], 1), torch.cat([v, _rows(st["va"]).float()], 1)
    q = _rows(st["q"]).float() / math.sqrt(d)
    # every rollout's rows against the history in one product, then each one's own keys
    qp = q.view(B, H, nq, d).transpose(0, 1).reshape(H, B * nq, d)
    lp = torch.bmm(qp, pk.transpose(1, 2).contiguous())
    lo = torch.bmm(q, k.transpose(1, 2).contiguous())
    hi = _shared_start(c) + (torch.arange(nq, device=DEV) // c["frame"] + 1) * c["frame"]
    lo.masked_fill_(~(c["n_prefix"] + torch.arange(n_own, device=DEV) < hi[:, None]), -math.inf)
    top = torch.maximum(lp.amax(2).view(H, B, nq).transpose(0, 1).reshape(B * H, nq),
                        lo.amax(2) if n_own else torch.full((B * H, nq), -math.inf, device=DEV))
    pp = lp.sub_(top.view(B, H, nq).transpose(0, 1).reshape(H, B * nq, 1)).exp_()
    po = lo.sub_(top[:, :, None]).exp_()
    back = lambda x: x.view(H, B, nq, -1).transpose(0, 1).reshape(B * H, nq, -1)  # noqa: E731
    total = back(pp.sum(2, keepdim=True)) + po.sum(2, keepdim=True)
    out = (back(torch.bmm(pp, pv)) + torch.bmm(po, v)) / total
    return out, top + total[:, :, 0].log()


# ------------------------------------------------------------ work and exact


def _token_bytes(c):
    ng = c["d"] // c["g"]
    v = c["d"] // 4 + 1 + (ng + 3) // 4 + (ng + 2 if c["storage"] & 1 else 2 * ng)
    return 2 * v + (c["r"] + 2 if c["r"] else 0)


def work(case):
    c = case
    B, H, d, r, e = c["batch"], c["heads"], c["d"], c["r"], 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rotary":
        values = 2 * B * H * c["n"] * d
        return dict(bytes=2 * values * e + (12 * B * c["n"] if c["explicit"] else 0), flops=3 * values)
    n_q, f = c["n_q"], c["frame"]
    block = 2 * c["kc"] * d * e + r * d * e
    if c["kind"] == "window":
        qs, ns, w, nk = c["q_start"], c["n_sink"], c["window"], c["n_cache"] + c["n_act"]
        pairs = corrected = 0
        for i in range(0, n_q, f):  # the rows of a frame see the same keys
            rows, hi = min(f, n_q - i), qs + i + f
            sink, low = min(ns, hi, nk), max(min(ns, hi), hi - w)
            pairs += rows * (sink + max(0, min(hi, nk) - low))
            corrected += rows * (min(sink, c["n_cache"]) + max(0, min(hi, c["n_cache"]) - low))
        low, high = max(ns, qs + f - w), qs + ((n_q - 1) // f + 1) * f
        packed = min(ns, c["n_cache"], high) + max(0, min(high, c["n_cache"]) - low)
        act = max(0, min(high, nk) - max(low, c["n_cache"])) + max(0, min(ns, nk, high) - c["n_cache"])
        read = packed * _token_bytes(c) + act * 2 * d * e + c["epochs"] * block
        return dict(bytes=B * H * (read + n_q * 2 * d * e), flops=B * H * (4 * d * pairs + 2 * r * corrected))
    npx, qs = c["n_prefix"], _shared_start(c)
    pairs = sum(min(f, n_q - i) * min(npx + c["n_cache"] + c["n_act"], qs + i + f) for i in range(0, n_q, f))
    read = npx * _token_bytes(c) + c["prefix_epochs"] * block
    mine = c["n_cache"] * _token_bytes(c) + c["n_act"] * 2 * d * e + block + n_q * 2 * d * e
    return dict(bytes=H * read + B * H * mine, flops=B * H * (4 * d + 2 * r) * pairs)


def _decode64(case, cache, bh, capacity, one, starts, n, tables):
    """One head's Keys, coefficients in place of their epoch's correction, and Values
    in 64 bits."""
    c, d = case, case["d"]
    keys, vals = [], []
    if n == 0:
        return [torch.empty(0, d, dtype=torch.float64, device=DEV) for _ in range(2)]
    for t, lo, hi in zip(tables, starts, starts[1:] + [n]):
        for side, to in (("k_", keys), ("v_", vals)):
            row = lambda name: _field(c, cache, bh, capacity, name)[one, lo:hi].contiguous()  # noqa: E731
            codes = row(side + "codes").int()
            q = torch.stack([codes % 4, codes // 4 % 4, codes // 16 % 4, codes // 64], 2).reshape(hi - lo, d).double()
            zb = row(side + "zp").int()
            z = torch.stack([zb % 4, zb // 4 % 4, zb // 16 % 4, zb // 64], 2).reshape(hi - lo, -1)[:, :d // c["g"]].double()
            s = row(side + "scale").double() * row(side + "sigma").view(torch.float16).double() if c["storage"] & 1 \
                else row(side + "scale").view(torch.float16).double()
            spread = lambda x: x.repeat_interleave(c["g"], 1)  # noqa: E731
            mu = t["mu_" + side[0]].view(bh, c["kc"], d)[one].double()
            to.append(mu[row(side + "ids")[:, 0].long()] + spread(s) * (q - spread(z)))
        if c["r"]:
            coef = row("k_coef").view(torch.int8).double() * row("k_cscale").view(torch.float16).double()
            keys[-1] = keys[-1] + coef @ t["u"].view(bh, c["r"], d)[one].double()
    return torch.cat(keys), torch.cat(vals)


def exact(case, seed):
    c, st = case, _inputs(case, seed)
    B, H, d, n_q = c["batch"], c["heads"], c["d"], c["n_q"] if "n_q" in c else c["n"]
    if c["kind"] == "rotary":
        return _exact_rotary(st)
    out = torch.zeros(B, n_q, H, d, dtype=torch.float64, device=DEV)
    lse = torch.full((B, H, n_q), -math.inf, dtype=torch.float64, device=DEV)
    window = c["kind"] == "window"
    start = c["q_start"] if window else _shared_start(c)
    end = start + (torch.arange(n_q, device=DEV) // c["frame"] + 1) * c["frame"]
    for b in range(B):
        for h in range(H):
            k, v = _decode64(c, st["cache"], B * H, c["n_cache"], b * H + h, st["starts"] if window else [0],
                             c["n_cache"], st["tables"])
            if not window:
                pk, pv = _decode64(c, st["prefix"], H, c["n_prefix"], h, st["starts"], c["n_prefix"], st["ptables"])
                k, v = torch.cat([pk, k]), torch.cat([pv, v])
            if c["n_act"]:
                k, v = torch.cat([k, st["ka"][b, :, h].double()]), torch.cat([v, st["va"][b, :, h].double()])
            at = torch.arange(k.shape[0], device=DEV)
            hide = at[None] >= end[:, None]
            if window:
                hide |= (at[None] >= c["n_sink"]) & (at[None] < end[:, None] - c["window"])
            lg = (st["q"][b, :, h].double() @ k.t().contiguous() * d ** -0.5).masked_fill_(hide, -math.inf)
            ls = torch.logsumexp(lg, 1)
            seen = ls > -math.inf
            lse[b, h] = ls
            out[b, seen, h] = (lg[seen] - ls[seen, None]).exp_() @ v
    return dict(out=out) if c["dtype"] == "bf16" else dict(out=out, lse=lse)


def _exact_rotary(st):
    """Each pair as a complex number times e^(i angle)."""
    c = st["case"]
    d, n = c["d"], c["n"]
    side = 2 * (d // 6)
    dims = [d - 2 * side, side, side]
    angle = []
    for b in range(c["batch"]):
        if st["pos"] is not None:
            place = [st["pos"][b, :, a].double() for a in range(3)]
        else:
            at = torch.arange(c["pos0"], c["pos0"] + n, device=DEV)
            place = [x.double() for x in (at // (c["gh"] * c["gw"]), at % (c["gh"] * c["gw"]) // c["gw"], at % c["gw"])]
        angle.append(torch.cat([p[:, None] * torch.exp(torch.arange(0, D, 2, device=DEV, dtype=torch.float64) *
                                                       (-math.log(c["base"]) / D)) for p, D in zip(place, dims)], 1))
    turn = torch.polar(torch.ones(1, 1, dtype=torch.float64, device=DEV), torch.stack(angle))[:, :, None]
    if c["inverse"]:
        turn = turn.conj()

    def one(x):
        x = x.double()
        if c["pairs"] == "adjacent":
            return torch.view_as_real(torch.view_as_complex(x.reshape(*x.shape[:3], d // 2, 2).contiguous()) * turn).reshape(x.shape)
        z = torch.complex(x[..., :d // 2], x[..., d // 2:]) * turn
        return torch.cat([z.real, z.imag], 3)

    return dict(q=one(st["q"]), k=one(st["k"]))
