"""quantwm_rotary against the turn in 64 bits (angles in extended precision): both
pairings, every axis split, grid and explicit positions up to 2^31, slices of a fused
projection, in place, odd sizes; the inverse as the gradient."""
import numpy as np
import pytest
import torch

from paper_2609_26425_amd import quantwm as qw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# batch, heads, d, tokens, dims, halves, dtype, explicit, first place or largest position, base
CASES = {
    "one-token": (1, 12, 128, 1, (44, 42, 42), False, "bf16", False, 12_345, 1e4),
    "chunk": (1, 40, 128, 333, (44, 42, 42), False, "bf16", False, 187_200, 1e4),
    "halves": (2, 3, 128, 77, (44, 42, 42), True, "bf16", True, 1000, 1e4),
    "time-only": (1, 2, 64, 50, (64, 0, 0), False, "f32", False, 100_000, 1e6),
    "width-only-halves": (1, 5, 64, 9, (0, 0, 64), True, "f32", True, 500, 1e4),
    "partial": (3, 7, 128, 31, (12, 2, 10), False, "bf16", True, 4000, 1e4),
    "partial-halves": (2, 5, 128, 31, (20, 8, 4), True, "f32", False, 3, 1e4),
    "partial-halves-bf16": (2, 5, 64, 31, (10, 22, 0), True, "bf16", False, 3, 1e4),
    "none": (1, 2, 64, 5, (0, 0, 0), False, "bf16", False, 9, 1e4),
    "far": (1, 2, 128, 40, (44, 42, 42), False, "f32", True, 2 ** 31 - 1, 1e4),
    "far-frames": (1, 2, 64, 40, (24, 20, 20), True, "f32", False, (2 ** 31 - 3) * 91, 1e4),
    "f32-odd": (2, 1, 64, 257, (24, 20, 20), False, "f32", False, 0, 1e4),
    "many": (4, 30, 128, 300, (44, 42, 42), False, "bf16", True, 90, 1e4),
}
GRID = (7, 13)


def _reference(x, place, dims, halves, base, sign):
    """The turn of x [B, n, H, d] (float64) by positions place [B, n, 3]."""
    axis = np.repeat(np.arange(3), [D // 2 for D in dims])
    # the frequencies as the library holds them (fp64), the angle in extended precision
    freq = np.array([float(base) ** (-2.0 * i / D) for D in dims for i in range(D // 2)])
    ang = place[..., axis].astype(np.longdouble) * freq.astype(np.longdouble)
    c, s = (np.asarray(f(ang), np.float64)[:, :, None] for f in (np.cos, np.sin))
    s = sign * s
    P = len(freq)
    out, x = x.copy(), x.astype(np.float64)
    a, b = (slice(0, P), slice(P, 2 * P)) if halves else (slice(0, 2 * P, 2), slice(1, 2 * P, 2))
    out = x.copy()
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., a] * s + x[..., b] * c
    size = np.zeros_like(x)  # |u| + |v| of each channel's pair
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return out, size


def _place(rng, B, n, explicit, at):
    if explicit:
        pos = rng.integers(max(0, at - 5000), at + 1, (B, n, 3))
        pos[0, 0] = at
        pos[-1, -1, 1] = -min(at, 5)  # positions may be negative
        return pos
    i = at + np.arange(n)
    area = GRID[0] * GRID[1]
    return np.repeat(np.stack([i // area, i // GRID[1] % GRID[0], i % GRID[1]], 1)[None], B, 0)


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("name", list(CASES))
def test_rotary(name, inverse):
    B, H, d, n, dims, halves, dtype, explicit, at, base = CASES[name]
    rng = np.random.default_rng(n + d + H)
    cfg = qw.make_config(B, H, d, 16, 16, 0, 1, 1, dtype)
    dt = cfg.torch_dtype
    axes = qw.rotary_axes(cfg, dims, *GRID, base=base, pairs=qw.ROTARY_HALVES if halves else qw.ROTARY_ADJACENT)
    qkv = torch.from_numpy(rng.standard_normal((B, n, 3, H, d))).to(DEV, dt)
    place = _place(rng, B, n, explicit, at)
    pos = torch.from_numpy(place.astype(np.int32)).to(DEV) if explicit else None
    pos0 = 0 if explicit else at
    # An angle is off by the fp64 roundings of the frequency (its power to an ulp, 2 pi,
    # the quotient) and of the product, 5 x 2^-53 of it, and by the fp32 remainder (2^-25
    # turns); sine and cosine by 2 ulp (2^-22); the two products and their sum by 3 x 2^-24.
    off = 5 * 2.0 ** -53 * float(np.abs(place).max()) + 2 * np.pi * 2.0 ** -25 + 2.0 ** -22 + 3 * 2.0 ** -24
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    want = [_reference(qkv[:, :, i].double().cpu().numpy(), place, dims, halves, base, -1.0 if inverse else 1.0) for i in (0, 1)]

    def good(got, i):
        ref, size = want[i]
        err = np.abs(got.double().cpu().numpy() - ref) - off * size - step * (np.abs(ref) + off * size)
        assert (err <= 0).all(), err.max()
        if 2 * (sum(dims) // 2) < d:
            assert torch.equal(got[..., sum(dims):], qkv[:, :, i][..., sum(dims):])

    outs = [torch.full((B, n, H, d), 7.0, dtype=dt, device=DEV) for _ in range(2)]
    qw.quantwm_rotary(cfg, axes, qkv[:, :, 0], qkv[:, :, 1], n, *outs, pos0=pos0, pos=pos, inverse=inverse)
    good(outs[0], 0)
    good(outs[1], 1)
    # contiguous, the Queries alone, and in place: the same bits
    q = qkv[:, :, 0].contiguous()
    alone = torch.full_like(q, 7.0)
    qw.quantwm_rotary(cfg, axes, q, None, n, alone, pos0=pos0, pos=pos, inverse=inverse)
    assert torch.equal(alone, outs[0])
    qw.quantwm_rotary(cfg, axes, q, None, n, q, pos0=pos0, pos=pos, inverse=inverse)
    assert torch.equal(q, outs[0])


@pytest.mark.parametrize("halves", [False, True])
def test_the_inverse_is_the_gradient(halves):
    """<g, d turn(x)> by differences along random directions equals <inverse(g), dx>."""
    cfg = qw.make_config(2, 3, 64, 16, 16, 0, 1, 1, "f32")
    axes = qw.rotary_axes(cfg, (24, 20, 4), *GRID, pairs=qw.ROTARY_HALVES if halves else qw.ROTARY_ADJACENT)
    gen = torch.Generator(device=DEV).manual_seed(1)
    R = lambda: torch.randn(2, 21, 3, 64, generator=gen, device=DEV)  # noqa: E731
    x, g = R(), R()

    def turn(t, inverse=False):
        out = torch.empty_like(t)
        qw.quantwm_rotary(cfg, axes, t.contiguous(), None, 21, out, pos0=1234, inverse=inverse)
        return out

    grad = turn(g, inverse=True)
    for _ in range(4):
        e = R()
        diff = ((turn(x + e).double() - turn(x - e).double()) / 2 * g.double()).sum()
        terms = (e.double().abs() * grad.double().abs()).sum() + (x.double().abs() * grad.double().abs()).sum()
        # every value within 2^-21 of its pair's size on either side; a pair's size is at most sqrt(2) of its norm
        assert abs(float(diff - (grad.double() * e.double()).sum())) <= 4 * 2.0 ** -21 * float(terms)
    back = turn(turn(x), inverse=True)
    assert (back - x).abs().max() <= 4 * 2.0 ** -21 * x.abs().max()


def test_given_frequencies():
    """freq replaces the powers of the base: with frequency pi / 2 a position turns a
    quarter, exactly up to the angle's rounding."""
    cfg = qw.make_config(1, 1, 64, 16, 16, 0, 1, 1, "f32")
    axes = qw.rotary_axes(cfg, (64, 0, 0), 1, 1, freq=[np.pi / 2] * 32)
    x = torch.randn(1, 4, 1, 64, device=DEV)
    out = torch.empty_like(x)
    qw.quantwm_rotary(cfg, axes, x, None, 4, out)
    want = x.clone()
    for t in (1, 2, 3):  # (u, v) -> (-v, u), t times
        for _ in range(t):
            u, v = want[:, t, :, 0::2].clone(), want[:, t, :, 1::2].clone()
            want[:, t, :, 0::2], want[:, t, :, 1::2] = -v, u
    assert (out - want).abs().max() <= 2.0 ** -21 * x.abs().max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("halves,dims", [(False, (2, 2, 6)), (False, (44, 42, 40)), (True, (12, 2, 18)), (False, (0, 0, 0))])
def test_channels_past_the_axes_are_copied(halves, dims, dtype):
    """bit for bit: the sign of a zero, and an infinity beside a finite channel."""
    cfg = qw.make_config(1, 3, 128, 16, 16, 0, 1, 1, dtype)
    axes = qw.rotary_axes(cfg, dims, *GRID, pairs=qw.ROTARY_HALVES if halves else qw.ROTARY_ADJACENT)
    x = torch.randn(1, 9, 3, 128, generator=torch.Generator().manual_seed(3)).to(cfg.torch_dtype)
    part = x[..., sum(dims):]
    part[..., 0], part[..., 1] = 1.5, -0.0
    part[:, ::2, :, 0], part[:, ::3, :, 1] = -0.0, float("inf")
    x = x.to(DEV)
    out = torch.full_like(x, 7.0)
    qw.quantwm_rotary(cfg, axes, x, None, 9, out, pos0=1000)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(out[..., sum(dims):].view(bits), x[..., sum(dims):].view(bits))
    assert out[..., : sum(dims)].isfinite().all()


def test_more_tokens_than_a_grid_dimension():
    """A workgroup a token, past 2^24 of them (34 GB, in place): the first and last tokens
    equal those of short calls."""
    cfg = qw.make_config(1, 16, 64, 16, 16, 0, 1, 1, "bf16")
    axes = qw.rotary_axes(cfg, (24, 20, 20), *GRID)
    n = (1 << 24) + 70_003
    if torch.cuda.mem_get_info()[0] < 3 * n * 16 * 64:
        pytest.skip("needs 50 GB of device memory")
    x = torch.empty(1, n, 16, 64, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(7)
    few = torch.randn(1, 9, 16, 64, generator=gen, device=DEV).bfloat16()
    at = [0, 65_530, (1 << 24) - 4, (1 << 24) + 65_531, n - 9]
    for i in at:
        x[:, i:i + 9] = few
    qw.quantwm_rotary(cfg, axes, x, None, n, x, pos0=11)
    for i in at:
        want = torch.empty_like(few)
        qw.quantwm_rotary(cfg, axes, few, None, 9, want, pos0=11 + i)
        assert torch.equal(x[:, i:i + 9], want)
