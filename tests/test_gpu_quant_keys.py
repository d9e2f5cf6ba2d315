"""Keys that are normed, turned and held in 8 bits, code by code and scale by
scale against the float64 oracle.

The kernel's key before it is rounded to a code: the norm is in 64 bits and
rounded to fp32 (E = 2^-24 of it, 2^-150 where fp32 is that coarse); the turn is
in 64 bits with a cosine and a sine that are off by 6 E (the angle 2 E, they
themselves 4 E) and is rounded to fp32 (E). So it lies within
t = (E + 2^-40) |y| + 2^-149 without a turn and 8 E m + 2^-148 with one, m what
the rotation can carry into the element. Rounding to codes and the choice of a
scale are monotone: code and scale lie between those of y - t and y + t, which
are one and the same away from a border.
"""
import numpy as np
import pytest

from oracle import heads as O
from helpers import dev, host
from test_gpu_heads import E, draw
from test_gpu_quant_cache import pool, values

pytestmark = pytest.mark.gpu


def codes_of(y, byte):
    """Rounded to codes of the rows' scale bytes."""
    f = np.exp2(byte.astype(np.float64) - 127)[..., None]
    z = y / f
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(z), 2.0 ** -30))), -6) - 3)
    return np.clip(np.rint(z / step) * step, -448, 448) * f


def bytes_of(top):
    return O.quantised(top[..., None])[1]


def held(B, x, gamma, eps, rot, dtype, positions=None):
    """(values, scale bytes) that a cache holds of keys x [T, H, D]."""
    import torch
    t, h, d = x.shape
    cfg = B.heads_config(h, h, d, dtype=dtype, norm=True, eps=eps, rot_dim=rot)
    w = {"gamma_k": None if gamma is None else dev(gamma, dtype), "freqs": B.rope_freqs(cfg) if rot else None}
    n = -(-t // 16)
    p = pool(n, h, 16, d)
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = B.PagedCache8(cfg, w, *p, torch.arange(n, **i32)[None], torch.tensor([t], **i32))
    k = dev(x, dtype)
    cache.append(k, k, cu_tokens=torch.tensor([0, t], **i32))
    torch.cuda.synchronize()
    rows = lambda a: a.transpose(0, 2, 1, *range(3, a.ndim)).reshape(n * 16, h, *a.shape[3:])[:t]  # noqa: E731
    return rows(values(p[0], p[2])), rows(p[2].cpu().numpy())


def reference(B, x, gamma, eps, rot, dtype):
    """(y, t) as above, tokens at rows 0 .. T - 1."""
    cfg = B.heads_config(1, 1, x.shape[-1], dtype=dtype, norm=True, eps=eps, rot_dim=rot)
    freqs = B.rope_freqs(cfg).cpu().numpy() if rot else np.zeros(0)
    ang = O.angles([np.arange(len(x))], freqs, (rot // 2,)) if rot else np.zeros((len(x), 0))
    with np.errstate(invalid="ignore"):  # zeros without eps, infinities
        y, m = O.norm_rope(x, gamma, float(np.float32(eps)), True, ang, rot, False)
    return y, (8 * E * m + 2.0 ** -148 if rot else (E + 2.0 ** -40) * np.abs(y) + 2.0 ** -149)


def check(got, byte, y, t, what):
    """Returns how many elements and scales lie next to a border."""
    nan = np.isnan(y)
    np.testing.assert_array_equal(np.isnan(got), nan, err_msg=str(what))
    y, t = np.where(nan, 0, y), np.where(nan, 0, t)
    small, large = (bytes_of(np.maximum(np.abs(y) + s * t, 0).max(-1)) for s in (-1, 1))
    assert ((small <= byte) & (byte <= large)).all(), (what, byte, small, large)
    lo, hi = codes_of(y - t, byte), codes_of(y + t, byte)
    z = np.where(nan, 0, got)
    bad = ~((lo <= z) & (z <= hi))
    assert not bad.any(), (what, int(bad.sum()), z[bad][:4], lo[bad][:4], hi[bad][:4])
    return int((lo != hi).sum()), int((small != large).sum())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-5])
def test_rows_of_far_magnitudes(gpu, dtype, d, eps):
    """Rows whose squares pass fp32's range on either side; infinities (the
    other elements of their rows become zeros), NaN, and rows of zeros."""
    rng = np.random.default_rng(1)
    # bf16 and fp32 alike end below 2^128 and begin above 2^-133
    powers = [0, 60, 62, 63, 64, 66, 80, 100, 123, -30, -60, -63, -64, -66, -75, -80, -100, -110]
    x = draw(rng, (len(powers) + 5, 2, d), dtype)
    x[:len(powers)] *= np.exp2(np.array(powers, np.float32))[:, None, None]
    x[-5, :, 5] = np.inf
    x[-4, 0, 3], x[-4, 1, d - 1] = -np.inf, np.inf
    x[-3, :, 7] = np.nan
    x[-2] = 0
    x[-1, :, 1:] = 0
    x = host(dev(x, dtype))
    g = host(dev(draw(rng, d, dtype, 0.25) + 1, dtype))
    for gamma in (None, g):
        for rot in (0, 32, d):
            check(*held(gpu, x, gamma, eps, rot, dtype), *reference(gpu, x, gamma, eps, rot, dtype), (gamma is None, rot))


@pytest.mark.parametrize("d", [64, 128])
def test_keys_next_to_borders(gpu, d):
    """Gains that bring a row's normed keys to within 0.6 to 2.6 fp32 steps of a
    border between two codes (a gain's step is at most two of the product's), and
    its top as near to one between two scales: more than the half step by which
    the kernel may be off, less than what a norm in 32 bits often is."""
    codes = np.arange(0x7F, dtype=np.uint8)
    e, f = codes >> 3, (codes & 7).astype(np.float64)
    grid = np.where(e > 0, (1 + f / 8) * np.exp2(e.astype(np.float64) - 7), f * 2.0 ** -9)
    rng = np.random.default_rng(2)
    for seed in range(24):
        x = draw(rng, (1, 1, d), "fp32", 3.0)
        x += np.sign(x)  # away from zero
        y = x[0, 0].astype(np.float64)
        y /= np.sqrt(np.mean(y * y))
        at = rng.integers(8, 126, d)  # normal codes
        border = (grid[at] + grid[at + 1 - (at == 126)]) / 2
        border[0] = 448
        side = rng.choice([-1, 1], d)
        gain = (border / np.abs(y)).astype(np.float32)
        for _ in range(4):
            away = side * (np.abs(y) * gain.astype(np.float64) - border)
            gain = np.where(away < 0.6 * np.spacing(border.astype(np.float32)),
                            np.nextafter(gain, np.where(side > 0, np.float32(np.inf), np.float32(0))), gain)
        away = side * (np.abs(y) * gain.astype(np.float64) - border) / np.spacing(border.astype(np.float32))
        assert (away >= 0.6).all()
        got, byte = held(gpu, x, gain, 0.0, 0, "fp32")
        want, want_byte = O.quantised(y * gain)
        assert byte[0, 0] == want_byte == (128 if side[0] > 0 else 127)
        np.testing.assert_array_equal(got[0, 0], want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hq, hk, d", [(32, 8, 128), (4, 2, 64), (16, 16, 64)])
def test_many_keys(gpu, dtype, hq, hk, d):
    """From 2,048 tokens on, with heads that fill a wave's passes (a token per
    wave) and that do not (four). An element in 2^11 may lie next to a border: 2 t
    over a step of 2^-4 |y| is 2^-16 m / |y|, and m / |y| is some ten in the mean."""
    import torch
    rng = np.random.default_rng(3)
    t = 2301
    cfg = gpu.heads_config(hq, hk, d, dtype=dtype, norm=True, eps=1e-5, rot_dim=d)
    g = host(dev(draw(rng, d, dtype, 0.25) + 1, dtype))
    w = {"gamma_q": dev(g, dtype), "gamma_k": dev(g, dtype), "freqs": gpu.rope_freqs(cfg)}
    n = -(-t // 16)
    p = pool(n, hk, 16, d)
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = gpu.PagedCache8(cfg, w, *p, torch.arange(n, **i32)[None], torch.tensor([t], **i32))
    x = {y: draw(rng, (t + 3, h, d), dtype) for y, h in (("q", hq), ("k", hk), ("v", hk))}
    q = dev(x["q"], dtype)
    q_out = torch.full_like(q, 5.0)
    cache.append(dev(x["k"], dtype), dev(x["v"], dtype), q=q, q_out=q_out, cu_tokens=torch.tensor([0, t], **i32))
    torch.cuda.synchronize()
    rows = lambda a: a.transpose(0, 2, 1, *range(3, a.ndim)).reshape(n * 16, hk, *a.shape[3:])  # noqa: E731
    k, kb, v, vb = rows(values(p[0], p[2])), rows(p[2].cpu().numpy()), rows(values(p[1], p[3])), rows(p[3].cpu().numpy())
    near, tops = check(k[:t], kb[:t], *reference(gpu, x["k"][:t], g, 1e-5, d, dtype), "keys")
    assert near <= t * hk * d / 2 ** 11 and tops <= t * hk / 2 ** 11, (near, tops)
    want, byte = O.quantised(x["v"][:t])
    np.testing.assert_array_equal(v[:t], want)
    np.testing.assert_array_equal(vb[:t], byte)
    for a, b in ((k, kb), (v, vb)):  # behind the last token, as they were
        assert np.isnan(a[t:]).all() and (b[t:] == 255).all()
    ang = O.angles([np.arange(t)], w["freqs"].cpu().numpy(), (d // 2,))
    ref, m = O.norm_rope(x["q"][:t], g, float(np.float32(1e-5)), True, ang, d, False)
    u = 2.0 ** -8 if dtype == "bf16" else E
    assert (np.abs(host(q_out)[:t] - ref) <= u * np.abs(ref) + 32 * E * m).all() and (q_out[t:] == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_scale_byte(gpu, dtype):
    """All codes under all scale bytes of 1..254: read back as the type rounds the
    value they stand for, which it holds exactly from 3 to 246. A token and a prompt
    that see one such row alone give its value as it is (bf16 takes weights in two
    terms, the second zero, so not past its largest value)."""
    import torch
    codes = torch.arange(256, dtype=torch.uint8).view(4, 64)
    n, i32 = 254 * 4, dict(dtype=torch.int32, device="cuda")
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    cfg = gpu.heads_config(1, 1, 64, dtype=dtype, norm=False, rot_dim=0)
    pages = codes.repeat(254, 1).view(n, 1, 1, 64).expand(-1, -1, 16, -1).contiguous().cuda()
    scales = torch.arange(1, 255, dtype=torch.uint8).repeat_interleave(4).view(n, 1, 1).expand(-1, -1, 16).contiguous().cuda()
    cache = lambda k, ks: gpu.PagedCache8(cfg, {}, k.view(torch.float8_e4m3fn), pages.view(torch.float8_e4m3fn), ks, scales,  # noqa: E731
                                          torch.arange(n, **i32)[:, None], torch.ones(n, **i32))
    value = codes.view(torch.float8_e4m3fn).double() * torch.exp2(torch.arange(1, 255).double() - 127)[:, None, None]
    want = value.to(dt)
    nan = torch.isnan(value)
    assert (want[2:246].double() == value[2:246])[~nan[2:246]].all()
    back = [torch.empty(n, 1, 64, dtype=dt, device="cuda") for _ in "kv"]
    cache(pages.clone(), scales.clone()).read(*back)
    flat = cache(torch.zeros_like(pages), torch.full_like(scales, 127))  # keys of zeros
    q = torch.ones(n, 1, 64, dtype=dt, device="cuda")
    token, prompt = flat.attend(q, 1), flat.attend(q, 1, cu_tokens=torch.arange(n + 1, **i32), max_new=32)
    for got, end in ((back[0], 254), (back[1], 254), (token, 246 if dtype == "bf16" else 254), (prompt, 254)):
        got = got.cpu().view(254, 4, 64)
        assert torch.isnan(got[nan]).all()
        ok = (got == want) | nan
        assert ok[:end].all(), [i + 1 for i in range(end) if not ok[i].all()]
