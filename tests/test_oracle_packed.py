"""Pins of the oracle's packed attention and 8-bit rows."""
import numpy as np

from oracle import heads as O


def inputs(t, hq, hk, d, seed):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal((t, h, d)) for h in (hq, hk, hk, hq)]


def test_against_the_paged_definition():
    """A sequence's tokens as its cache: the same rows seen, the same results."""
    q, k, v, _ = inputs(40, 4, 2, 8, 1)
    cu = [0, 13, 13, 40]
    for window, sinks in ((0, 0), (5, 2)):
        out, lse, err, mag = O.packed_attention(q, k, v, cu, 0.3, window, sinks)
        for s, (a, b) in enumerate(zip(cu[:-1], cu[1:])):
            if a == b:
                continue
            pages = [x[a:b].transpose(1, 0, 2)[None] for x in (k, v)]
            ref = O.paged_attention(q[a:b], *pages, np.zeros((1, 1), int), [b - a], [0, b - a], 0.3, window, sinks)
            for x, y in zip((out, lse, err, mag), ref):
                np.testing.assert_allclose(x[a:b], y, rtol=1e-12, atol=1e-14)


def test_gradients_against_differences():
    q, k, v, do = inputs(21, 6, 2, 8, 2)
    cu, h = [0, 9, 20], 1e-6  # a token behind the last sequence
    for window, sinks in ((0, 0), (4, 1)):
        grads, _ = O.packed_attention_backward(q, k, v, do, cu, 0.4, window, sinks)
        f = lambda *x: np.nansum(O.packed_attention(*x, cu, 0.4, window, sinks)[0] * do)  # noqa: E731
        rng = np.random.default_rng(3)
        for i in range(3):
            along = rng.standard_normal((q, k, v)[i].shape)
            ends = [f(*(x + s * h * along if j == i else x for j, x in enumerate((q, k, v)))) for s in (1, -1)]
            np.testing.assert_allclose((ends[0] - ends[1]) / (2 * h), (grads[i] * along).sum(), rtol=1e-6, atol=1e-7)
            assert not grads[i][20:].any()


def test_one_row_has_no_score_gradient():
    q, k, v, do = inputs(3, 2, 1, 8, 4)
    (dq, dk, dv), _ = O.packed_attention_backward(q, k, v, do, [0, 1, 2, 3], 0.5)
    assert np.abs(dq).max() < 1e-14 and np.abs(dk).max() < 1e-14
    np.testing.assert_allclose(dv[:, 0], do.sum(1))


def test_rows_of_8_bits():
    """Against the type's own conversion, at every code, between codes and past
    them; the scale's edges by hand."""
    import torch
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    codes = codes[np.isfinite(codes)]
    mid = np.sort(codes[codes >= 0])
    points = np.concatenate([mid, (mid[1:] + mid[:-1]) / 2, mid[:-1] * 0.75 + mid[1:] * 0.25, [448.0]])
    row = np.concatenate([points, -points])[None]
    got, byte = O.quantised(row)
    assert byte[0] == 127
    want = torch.from_numpy(row).float().to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(got, want)
    for top, e in ((448.0, 0), (448.0001, 1), (224.0, -1), (224.0001, 0), (1.0, -8), (0.0, -110), (2.0 ** -120, -110)):
        assert O.quantised(np.array([[top, -top / 3]]))[1][0] == e + 127, top
    got, byte = O.quantised(np.array([[np.inf, 1.0, np.nan, -2.0]]))
    assert byte[0] == 127 - 7 and np.isnan(got[0, [0, 2]]).all() and got[0, 1] == 1 and got[0, 3] == -2
