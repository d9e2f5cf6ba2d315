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
