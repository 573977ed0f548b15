"""The few-row attention kernels at the ends of their operands' ranges, and which of the
two kernels a launch takes: against a plain 64-bit softmax over the Keys in one form only
(as they decode for the few-row kernel, rounded to BF16 for the tiles), not in either."""
import numpy as np
import pytest
import torch

import oracle
import stream64 as s64
from paper_2609_26425_amd import quantwm as qw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def stream(rng, n, keys, mu, starts=(0,), batch=1, heads=2, d=128, kc=16, g=32, r=8, st=0, values=None, mu_v=None):
    """n packed BF16 tokens: keys(rng, tables' mu_k, tokens) of tables mu(rng), Values likewise
    (standard normal without `values`)."""
    p = s64.Packed(rng, batch, heads, d, kc, g, r, "bf16", st, [0], 0, capacity=n)
    p.n, p.starts, p.tables = n, list(starts), []
    normal = lambda *s: rng.standard_normal(s)  # noqa: E731
    for lo, hi in zip(p.starts, p.starts[1:] + [n]):
        mk = s64.rounded(mu(rng, (batch, heads, kc, d)), "bf16")
        mv = s64.rounded((mu_v or (lambda rng, s: normal(*s)))(rng, (batch, heads, kc, d)), "bf16")
        u = np.stack([np.linalg.qr(normal(d, d))[0][:r] for _ in range(batch * heads)]).reshape(batch, heads, r, d)
        t = (mk, mv, np.ones((batch, heads, d), np.float32), s64.rounded(u, "bf16"), np.ones((batch, heads, r), np.float32))
        k = s64.rounded(keys(rng, mk, (batch, hi - lo, heads, d)), "bf16")
        v = s64.rounded(normal(batch, hi - lo, heads, d) if values is None else values(rng, mv, (batch, hi - lo, heads, d)), "bf16")
        oracle.append(p.ocfg, t, p.cache, lo, k, v)
        p.tables.append(t)
    return p


def normal(size):
    """Keys and tables of that size."""
    return dict(keys=lambda rng, mk, s: size * rng.standard_normal(s), mu=lambda rng, s: size * rng.standard_normal(s))


def members(rng, mu, s):
    """Tokens that are centroids themselves: no residual."""
    batch, n, heads, d = s
    z = rng.integers(0, mu.shape[2], (batch, n, heads))
    return mu[np.arange(batch)[:, None, None], np.arange(heads), z]


def seen(n, n_q):
    return np.arange(n) <= (n - n_q + np.arange(n_q))[:, None]


def window(p, q, few, ka=None, va=None, workspace=True):
    """quantwm_attend_window over everything, the Queries last: against the given form of
    the Keys. Returns the results, and whether the other form fits too."""
    B, n_q = q.shape[:2]
    n_act = 0 if ka is None else ka.shape[1]
    n = p.n + n_act
    k, v = p.keys_values()
    if n_act:
        k, v = (np.concatenate([x, y.transpose(0, 2, 1, 3)], 2) for x, y in ((k, ka), (v, va)))
    visible = seen(n, n_q)
    refs = {}
    for form in (False, True):
        lg = p.logits(q, form)
        if n_act:
            lg = np.concatenate([lg, s64.exact_logits(q, ka)], 3)
        refs[form] = (*s64.softmax(lg, visible, v), s64.tolerances(q, k, n, p.r, "bf16", p.residuals() if form else None))
    nb = qw.quantwm_attend_window_workspace_bytes(p.cfg, p.n, n_act, n_q, 1, 0, n) if workspace else 0
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV) if nb else None
    qd = s64.dev(q, torch.bfloat16)
    kd, vd = (s64.dev(x, torch.bfloat16) if n_act else None for x in (ka, va))
    out, lse = torch.full_like(qd, 7.0), torch.full((B, p.heads, n_q), 7.0, device=DEV)
    qw.quantwm_attend_window(p.cfg, p.blocks(), p.starts, p.on_device(), p.n, kd, vd, n_act, qd, n_q, n - n_q, 1, 0, n,
                             out, lse, ws)
    torch.cuda.synchronize()
    s64.check(out, lse, *refs[few])
    try:
        s64.check(out, lse, *refs[not few])
    except AssertionError:
        return out, lse, False
    return out, lse, True


def queries(rng, p, size, n_q, peaks=2.0):
    """Queries of which three in four have most of their weight on one key."""
    q = 0.5 / size * rng.standard_normal((p.batch, n_q, p.heads, p.d))
    k = p.keys_values()[0]
    for i in range(n_q):
        if i % 4 != 3:
            q[:, i] += peaks / size ** 2 * k[:, :, (37 * i + 5) % p.n]
    return s64.rounded(q, "bf16")


# Keys' size: steps from a few units of the last place of binary16's smallest values to such
# that three of them pass its largest
SIZES = [2.0 ** -23, 2.0 ** -20, 2.0 ** -18, 2.0 ** -16, 2.0 ** -14, 2.0 ** -12, 6000.0, 20000.0]
SHAPES = {  # packed, exact keys, Queries, head_dim, group, rank, storage
    "one": (1500, 0, 1, 128, 32, 8, 0), "one-act": (700, 9, 1, 64, 16, 4, 0), "some": (6500, 0, 16, 128, 16, 16, 0),
    "wide": (7400, 3, 20, 64, 64, 0, 0), "wide-128": (7400, 0, 20, 128, 32, 32, 0), "some-i8": (1500, 0, 4, 128, 32, 8, 1),
}


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_key_steps_of_any_size(shape, size):
    n, n_act, n_q, d, g, r, st = SHAPES[shape]
    rng = np.random.default_rng(n + int(np.log2(size)) % 64)
    p = stream(rng, n, **normal(size), d=d, g=g, r=r, st=st)
    res = np.abs(p.residuals())
    assert res.max() > 65504.0 if size > 1e4 else size > 1 or st or 0 < res.max() < 8 * size  # at most three steps
    q = queries(rng, p, size, n_q)
    ka, va = (s64.rounded(x * rng.standard_normal((1, n_act, 2, d)), "bf16") if n_act else None for x in (size, 1.0))
    window(p, q, True, ka, va)


def test_key_steps_of_two_sizes_in_one_chunk():
    """Every other token's steps times 3 pass binary16's range in the first channels; the
    others are of size 1."""
    rng, n, d = np.random.default_rng(1), 1500, 128
    big = np.where(np.arange(d) < 64, 20000.0, 1.0)

    def keys(rng, mk, s):
        return rng.standard_normal(s) * np.where((np.arange(s[1]) % 2 == 0)[None, :, None, None], big, np.where(big > 1, 0, 1.0))

    def mu(rng, s):
        return rng.standard_normal(s) * np.where((np.arange(s[2]) % 2 == 0)[:, None], big, np.where(big > 1, 0, 1.0))
    for n_q in (1, 3):
        p = stream(rng, n, keys, mu)
        q = s64.rounded(0.5 / np.where(big > 1, big, 1.0) * rng.standard_normal((1, n_q, 2, d)), "bf16")
        window(p, q, True)


@pytest.mark.parametrize("size", [2.0 ** -20, 2.0 ** -16, 20000.0])
def test_shared_key_steps_of_any_size(size):
    B, H, d, n_pre, n_own, n_q = 3, 2, 128, 1500, 700, 1
    rng = np.random.default_rng(int(np.log2(size)) % 64)
    pre, own = stream(rng, n_pre, **normal(size)), stream(rng, n_own, **normal(size), batch=B, g=16, r=4)
    q = queries(rng, own, size, n_q)
    q[1] = queries(rng, pre, size, n_q)[0]
    (pk, pv), (k, v), flat = pre.keys_values(), own.keys_values(), q.reshape(1, B * n_q, H, d)
    k, v = (np.concatenate([np.repeat(x, B, 0), y], 2) for x, y in ((pk, k), (pv, v)))
    n = n_pre + n_own
    lg = np.concatenate([pre.logits(flat, True).reshape(H, B, n_q, n_pre).transpose(1, 0, 2, 3), own.logits(q, True)], 3)
    res = np.concatenate([np.repeat(pre.residuals(), B, 0), own.residuals()], 2)
    ref = (*s64.softmax(lg, np.ones((n_q, n), bool), v), s64.tolerances(q, k, 2 * n + 64, 8, "bf16", res))
    ws = torch.empty(qw.quantwm_attend_shared_workspace_bytes(pre.cfg, n_pre, own.cfg, n_own, 0, n_q), dtype=torch.uint8, device=DEV)
    qd = s64.dev(q, torch.bfloat16)
    out, lse = torch.full_like(qd, 7.0), torch.empty(B, H, n_q, device=DEV)
    qw.quantwm_attend_shared(pre.cfg, pre.blocks(), [0], pre.on_device(), n_pre, own.cfg, own.blocks(), own.on_device(), n_own,
                             None, None, 0, qd, n_q, n - 1, 1, out, lse, ws)
    torch.cuda.synchronize()
    s64.check(out, lse, *ref)


@pytest.mark.parametrize("power,small", [(60, -60), (118, -118), (114, -86), (118, -90), (125, -97)])
@pytest.mark.parametrize("n_q,few", [(1, True), (3, True), (20, True), (40, False)])
def test_large_key_tables(power, small, n_q, few):
    """Key centroids far out, and Queries as small or logits as large: all finite."""
    rng = np.random.default_rng(power + n_q)
    p = stream(rng, 7400 if n_q == 20 else 900, members, lambda rng, s: rng.uniform(-1.5, 1.5, s), r=4)
    assert not p.residuals().any()  # so the packed tokens are those of the scaled tables too
    p.tables = [(np.ldexp(t[0], power), *t[1:]) for t in p.tables]
    q = s64.rounded(np.ldexp(0.5 * rng.standard_normal((1, n_q, 2, 128)), small), "bf16")
    visible = seen(p.n, n_q)
    lg = np.where(visible, p.logits(q, few), -np.inf)
    top = lg.max(-1, keepdims=True)
    first = lg > top - 2.0 ** -30 * np.abs(top)  # the best centroid's tokens
    out, lse, _ = window(p, q, few)
    assert out.isfinite().all() and lse.isfinite().all()
    if power + small > 0:  # the mean Value of those tokens, where they lead by more than the logits err
        qk = np.matmul(np.abs(q).transpose(0, 2, 1, 3), np.abs(p.keys_values()[0]).transpose(0, 1, 3, 2)).max() / 128 ** 0.5
        led = top[..., 0] - np.where(first, -np.inf, lg).max(-1) > 4 * 140 * 2.0 ** -24 * qk + 100
        assert led.mean() > 0.9
        ref, _, mag = s64.softmax(np.where(first, 0.0, -np.inf), visible, p.keys_values()[1])
        # their weights are equal: half a step of the result, and the sum's order
        err = np.abs(out.double().cpu().numpy() - ref) - 2.0 ** -8 * np.abs(ref) - p.n * 2.0 ** -23 * mag
        assert (err[led.transpose(0, 2, 1)] <= 0).all()


@pytest.mark.parametrize("power", [-90, -108, -112, -116, -120])
@pytest.mark.parametrize("n_q,few", [(1, True), (20, True), (40, False)])
@pytest.mark.parametrize("steps", [False, True])
def test_small_value_tables(steps, power, n_q, few):
    """Value centroids near the smallest normal numbers, and Values that are centroids, or
    residuals of size 1 upon them."""
    rng = np.random.default_rng(-power + n_q)
    n = 7400 if n_q == 20 else 300
    p = stream(rng, n, **normal(1.0), values=None if steps else members, mu_v=lambda rng, s: 1.0 + np.abs(rng.standard_normal(s)))
    p.tables = [(t[0], np.ldexp(t[1], power), *t[2:]) for t in p.tables]
    q = s64.rounded(rng.standard_normal((1, n_q, 2, 128)), "bf16")
    window(p, q, few)


# packed, exact keys, Queries, epochs' starts, rank, storage, with a workspace: whether the
# few-row kernel takes the launch
LAUNCHES = {
    "one": (True, 900, 0, 1, [0], 8, 0, True), "one-unsplit": (True, 900, 0, 1, [0], 8, 0, False),
    "one-of-few-keys": (True, 40, 0, 1, [0], 4, 1, True), "one-act": (True, 900, 70, 1, [0], 0, 0, True),
    "two-parts-at-least": (False, 900, 70, 1, [0], 0, 0, False), "epochs": (True, 900, 9, 3, [0, 64, 200], 12, 1, True),
    "many-epochs": (False, 2700, 20, 7, [66 * i for i in range(40)], 4, 0, True),
    "many-epochs-19": (True, 7200, 20, 19, [180 * i for i in range(40)], 4, 0, True),
    "sixteen": (True, 5760, 0, 16, [0], 16, 0, True), "sixteen-of-fewer-keys": (False, 5759, 0, 16, [0], 16, 0, True),
    "wide": (True, 11_904, 0, 32, [0], 4, 0, True), "wide-of-fewer-keys": (False, 11_903, 0, 32, [0], 4, 0, True),
    "two-blocks": (False, 13_000, 0, 33, [0], 4, 0, True), "odd-rank": (False, 900, 0, 1, [0], 13, 0, True),
    "even-rank": (False, 900, 0, 1, [0], 6, 1, True),
}


@pytest.mark.parametrize("name", list(LAUNCHES))
def test_which_kernel_takes_a_launch(name):
    """Keys around a far point common to all, which cancels in the softmax: rounded to BF16
    they lose a good part of what tells them apart, so only one of the forms fits the results."""
    few, n, n_act, n_q, starts, r, st, ws = LAUNCHES[name]
    rng, H, d = np.random.default_rng(n + n_q + r), 2, 64
    far = 512.0 * rng.choice([-1.0, 1.0], (H, d))
    p = stream(rng, n, lambda rng, mk, s: far + 4 * rng.standard_normal(s), lambda rng, s: far[:, None] + 4 * rng.standard_normal(s),
               starts=starts, heads=H, d=d, kc=16, g=32, r=r, st=st)
    q = s64.rounded(0.25 * rng.standard_normal((1, n_q, H, d)), "bf16")
    ka, va = (s64.rounded(x + rng.standard_normal((1, n_act, H, d)), "bf16") if n_act else None for x in (far, 0.0))
    _, _, either = window(p, q, few, ka, va, ws)
    assert not either
