"""Pins of the heads oracle: what a rotation keeps, gradients against central
differences, the attention against closed forms, rows and pages by hand."""
import numpy as np
import pytest

from oracle import heads as O

AXES = {"one": (16,), "two": (5, 11), "three": (3, 1, 12)}


def setup(seed, t=3, h=2, d=64, rot=32, axes=(16,)):
    rng = np.random.default_rng(seed)
    freqs = 10000.0 ** (-np.arange(rot // 2) / (rot // 2))
    pos = rng.integers(0, 1000, (len(axes), t))
    return rng, rng.standard_normal((t, h, d)), 1 + 0.1 * rng.standard_normal(d), O.angles(pos, freqs, axes), pos, freqs


@pytest.mark.parametrize("style", [False, True])
@pytest.mark.parametrize("axes", AXES.values(), ids=AXES.keys())
def test_rotation_keeps_lengths_and_relative_positions(style, axes):
    _, x, gamma, ang, pos, freqs = setup(1, axes=axes)
    y, mag = O.norm_rope(x, gamma, 1e-6, True, ang, 32, style)
    z = x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * gamma
    assert np.allclose((y * y).sum(-1), (z * z).sum(-1)) and np.array_equal(y[..., 32:], z[..., 32:])
    assert (np.abs(y) <= mag + 1e-12).all()
    moved, _ = O.norm_rope(x, gamma, 1e-6, True, O.angles(pos + 77, freqs, axes), 32, style)
    assert np.allclose(np.einsum("thd,shd->tsh", y, y), np.einsum("thd,shd->tsh", moved, moved))


def test_a_pair_by_hand():
    x = np.arange(64, dtype=float)[None, None]
    for style, (a, b) in ((False, (1, 9)), (True, (2, 3))):
        y, _ = O.norm_rope(x, None, 0.0, False, np.full((1, 8), 0.3), 16, style)
        c, s = np.cos(0.3), np.sin(0.3)
        assert np.isclose(y[0, 0, a], a * c - b * s) and np.isclose(y[0, 0, b], a * s + b * c)


@pytest.mark.parametrize("style", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_gradients_against_central_differences(style, norm):
    rng, x, gamma, ang, _, _ = setup(2)
    dy = rng.standard_normal(x.shape)
    dx, dg, _, _ = O.norm_rope_backward(x, gamma, 1e-3, norm, ang, 32, style, dy)

    def loss(x, gamma):
        return (O.norm_rope(x, gamma, 1e-3, norm, ang, 32, style)[0] * dy).sum()

    e = 1e-5
    for at in [(0, 0, 0), (1, 1, 20), (2, 0, 40), (2, 1, 63)]:
        d = np.zeros_like(x)
        d[at] = e
        assert np.isclose((loss(x + d, gamma) - loss(x - d, gamma)) / (2 * e), dx[at], atol=1e-7)
        if norm:
            d = np.zeros_like(gamma)
            d[at[2]] = e
            assert np.isclose((loss(x, gamma + d) - loss(x, gamma - d)) / (2 * e), dg[at[2]], atol=1e-7)


def test_rows_and_places():
    assert O.token_rows([5, 0, 3], [0, 2, 2, 5]) == [(0, 3), (0, 4), (2, 0), (2, 1), (2, 2)]
    assert O.token_rows([5, 0], None) == [(0, 4), (1, -1)]
    table = [7, -1, 9]
    assert O.place(table, 17, 16, 8) is None and O.place(table, 3, 16, 8) == (7, 3)
    assert O.place(table, 33, 16, 8) is None and O.place(table, 33, 16, 10) == (9, 1)
    assert O.place(table, -1, 16, 8) is None and O.place(table, 48, 16, 10) is None
    assert list(np.nonzero(O.visible(9, 12, 3, 2))[0]) == [0, 1, 7, 8, 9]
    assert list(np.nonzero(O.visible(1, 12, 3, 2))[0]) == [0, 1]
    assert O.visible(9, 12, 0, 2).sum() == 10


def test_attention_closed_forms():
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((6, 2, 16, 64)), rng.standard_normal((6, 2, 16, 64))
    table = np.array([[4, 0, 5], [2, 1, -1], [3, 3, 3]])
    q = rng.standard_normal((3, 4, 64))
    # no scale: the mean of the visible values, and the count in lse
    out, lse, _, _ = O.paged_attention(q, k, v, table, [37, 20, 0], None, 0.0, 10, 2)
    rows = [0, 1] + list(range(27, 37))
    want = np.stack([v[table[0][j // 16], :, j % 16] for j in rows]).mean(0)
    assert np.allclose(out[0], np.repeat(want, 2, 0)) and np.allclose(lse[0], np.log(12))
    assert (out[2] == 0).all() and np.isneginf(lse[2]).all()
    # one visible row: that row's value; a huge score alone decides
    out, lse, _, _ = O.paged_attention(q, k, v, table, [37, 20, 1], None, 0.3, 1, 0)
    assert np.allclose(out[1], np.repeat(v[1, :, 3], 2, 0)) and np.allclose(lse[1, 3], 0.3 * k[1, 1, 3] @ q[1, 3])
    # a prompt equals its tokens one by one
    both, _, _, _ = O.paged_attention(q, k, v, table, [37, 20, 0], [0, 1, 3, 3], 0.2)
    one, _, _, _ = O.paged_attention(q[1:2], k, v, table[1:2], [19], None, 0.2)
    assert np.allclose(both[1], one[0])
    # a token behind the last sequence
    assert np.isnan(O.paged_attention(q, k, v, table, [37, 20, 0], [0, 1, 2, 2], 0.2)[0][2]).all()
