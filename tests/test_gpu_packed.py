"""Attention over packed sequences on the GPU, forward and backward, against the
float64 oracle.

Tolerances, per element, from the roundings that can occur (u: half a step of
the result's type, 2^-8 of it in bf16 and 2^-24 in fp32; E = 2^-24; w: half a
step of a weight in bf16 products, 2^-8, none in fp32; n rows seen at most):
* forward: u |o| + (2 d + (n + 64) E + w) m, m = sum p |v|. d, a score's error:
  (D + 10) E s + 8 E, s the largest sum of |q||k| terms times the scale.
* lse: 2 d + (n + 64) E + 4 E |lse|.
* the backward forms a weight again from its score (d), the log-sum (above) and
  an exponential (8 E, and 2 E of its argument, below |lse| + s): its relative
  error. out is off by the forward's tolerance, a product of D terms by (D + 10) E
  of their magnitudes; the oracle carries these to the gradients
  (packed_attention_backward), whose sums of N terms add (N + 64) E of their
  magnitudes, and the last rounding u. A weight below 2^-126 may be zero in
  fp32, and with it what it weighs: 2^-126 of |dO| in dV, of |dO| (|v| + |O|)
  over D channels times the scale and |k| or |q| in the others, N times.
"""
import numpy as np
import pytest

from oracle import heads as O
from helpers import dev, host
from test_gpu_heads import E, U, close, draw, laid_out

pytestmark = pytest.mark.gpu

CASES = {
    # name: (lengths, heads, kv heads, head_dim, dtype, window, sinks, layout, tokens behind)
    "one_token": ([1], 4, 2, 64, "bf16", 0, 0, "plain", 0),
    "ones_and_none": ([1, 0, 1, 2, 0], 3, 3, 128, "fp32", 0, 0, "plain", 3),
    "block_edges": ([31, 32, 33, 63, 64, 65], 4, 4, 64, "bf16", 0, 0, "band", 1),
    "workgroup_edges": ([127, 0, 128, 129, 257], 2, 1, 128, "bf16", 0, 0, "heads", 70),
    "group_of_5": ([200, 3, 77], 5, 1, 64, "bf16", 0, 0, "plain", 0),
    "group_of_16": ([150, 41], 16, 1, 128, "bf16", 0, 0, "band", 2),
    "group_of_40_fp32": ([70], 40, 1, 64, "fp32", 0, 0, "plain", 0),
    "window_1": ([100, 5], 2, 2, 64, "bf16", 1, 0, "plain", 0),
    "window_1_sinks_fp32": ([140], 4, 2, 128, "fp32", 1, 3, "plain", 0),
    "window_33_sinks_40": ([300, 10], 6, 2, 64, "bf16", 33, 40, "heads", 0),
    "window_130_sinks_130": ([500], 4, 4, 128, "bf16", 130, 130, "plain", 0),
    "window_200_fp32": ([290, 290], 4, 1, 64, "fp32", 200, 0, "band", 5),
    "window_past_all": ([90, 20], 2, 1, 64, "bf16", 1 << 40, 1 << 40, "plain", 0),
    "long": ([1111], 2, 1, 64, "bf16", 0, 0, "plain", 0),
    "long_fp32": ([700, 33], 2, 2, 128, "fp32", 0, 0, "heads", 0),
}


def inputs(name, seed=1, loud=1.5):
    lens, hq, hk, d, dtype, window, sinks, layout, behind = CASES[name]
    rng = np.random.default_rng(seed)
    t = sum(lens) + behind
    x = {n: draw(rng, (t, h, d), dtype, s) for n, h, s in (("q", hq, loud), ("k", hk, 1), ("v", hk, 1), ("do", hq, 1))}
    x["cu"] = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    return x


def on_gpu(B, name, x):
    import torch
    lens, hq, hk, d, dtype, window, sinks, layout, behind = CASES[name]
    g = {n: laid_out(x[n], dtype, layout) for n in ("q", "k", "v", "do")}
    g["cu"] = torch.from_numpy(x["cu"]).cuda()
    g["cfg"] = B.heads_config(hq, hk, d, dtype=dtype, norm=False, rot_dim=0)
    g["kw"] = dict(window=window, sinks=sinks)
    g["most"] = max(lens)
    return g


def forward(B, g, **kw):
    return B.packed_attention_forward(g["cfg"], g["q"], g["k"], g["v"], g["cu"], g["most"], **g["kw"], **kw)


def backward(B, g, out, lse, **kw):
    return B.packed_attention_backward(g["cfg"], g["q"], g["k"], g["v"], out, lse, g["do"], g["cu"], g["most"], **g["kw"], **kw)


def tolerances(name, ref):
    """(of out, of lse, a recomputed weight's relative error)."""
    lens, hq, hk, d, dtype, window, sinks, layout, behind = CASES[name]
    out, lse, err, mag = ref
    n, w = max(lens), 2.0 ** -8 if dtype == "bf16" else 0.0
    s = (d + 10) * E * err + 8 * E
    of_lse = 2 * s + (n + 64) * E + 4 * E * np.abs(lse)
    of_out = U[dtype] * np.abs(out) + ((2 * s + (n + 64) * E + w)[..., None]) * mag
    return of_out, of_lse, s + of_lse + 8 * E + 2 * E * (np.abs(lse) + err)


def check_backward(name, x, got, ref, scale):
    lens, hq, hk, d, dtype, window, sinks, layout, behind = CASES[name]
    of_out, _, of_weight = tolerances(name, ref)
    w = 2.0 ** -8 if dtype == "bf16" else 0.0
    n = max(lens)
    sums = (n * (hq // hk) + 64) * E
    grads, bounds = O.packed_attention_backward(x["q"], x["k"], x["v"], x["do"], x["cu"], scale, window, sinks, of_out,
                                                of_weight + sums, w, (d + 10) * E + sums)
    t = x["cu"][-1]
    most = {y: float(np.abs(x[y]).max()) for y in ("q", "k", "v", "do")}
    lost = 2.0 ** -126 * n * (hq // hk) * most["do"]  # by weights that are zero
    lost_ds = lost * 2 * d * most["v"] * abs(scale)
    for what, a, b, tol, zero in zip(("dq", "dk", "dv"), got, grads, bounds, (lost_ds * most["k"], lost_ds * most["q"], lost)):
        close(host(a)[:t], b[:t], U[dtype] * np.abs(b[:t]) + (1 + U[dtype]) * tol[:t] + zero, (name, what))


@pytest.mark.parametrize("name", CASES)
def test_forward_and_backward(gpu, name):
    import torch
    x = inputs(name)
    g = on_gpu(gpu, name, x)
    lens, hq, hk, d, dtype, window, sinks, layout, behind = CASES[name]
    out, lse = forward(gpu, g)
    got = backward(gpu, g, out, lse)
    torch.cuda.synchronize()
    ref = O.packed_attention(x["q"], x["k"], x["v"], x["cu"], d ** -0.5, window, sinks)
    t = x["cu"][-1]
    of_out, of_lse, _ = tolerances(name, ref)
    close(host(out)[:t], ref[0][:t], of_out[:t], (name, "out"))
    close(host(lse)[:t], ref[1][:t], of_lse[:t], (name, "lse"))
    for y in (out, lse, *got):  # poisoned before the call
        assert torch.isnan(y[t:]).all()
    check_backward(name, x, got, ref, d ** -0.5)
    again = backward(gpu, g, *forward(gpu, g))
    assert all(torch.equal(a[:t], b[:t]) for a, b in zip(got, again))


@pytest.mark.parametrize("name", ["workgroup_edges", "window_200_fp32", "group_of_5"])
@pytest.mark.parametrize("loud, scale", [(30.0, None), (2.0, -0.3), (1.0, 0.0)])
def test_sharp_flat_and_turned_weights(gpu, name, loud, scale):
    """Scores of hundreds, a negative scale, and none at all."""
    lens, hq, hk, d, dtype, window, sinks, layout, behind = CASES[name]
    x = inputs(name, 2, loud)
    g = on_gpu(gpu, name, x)
    f = d ** -0.5 if scale is None else scale
    out, lse = forward(gpu, g, scale=scale)
    got = backward(gpu, g, out, lse, scale=scale)
    ref = O.packed_attention(x["q"], x["k"], x["v"], x["cu"], f, window, sinks)
    t = x["cu"][-1]
    of_out, of_lse, _ = tolerances(name, ref)
    close(host(out)[:t], ref[0][:t], of_out[:t], name)
    close(host(lse)[:t], ref[1][:t], of_lse[:t], name)
    check_backward(name, x, got, ref, f)


@pytest.mark.parametrize("name", ["ones_and_none", "window_1_sinks_fp32", "long_fp32"])
def test_backward_against_differences(gpu, name):
    """The gradients along a direction against a central difference of the
    forward's results in fp32. The difference's own error is its distance in
    float64 and the forward's roundings over the step."""
    lens, hq, hk, d, dtype, window, sinks, layout, behind = CASES[name]
    x = inputs(name, 3)
    t, h = x["cu"][-1], 2.0 ** -6
    g = on_gpu(gpu, name, x)
    got = [host(y) for y in backward(gpu, g, *forward(gpu, g))]
    rng = np.random.default_rng(4)
    for i, n in enumerate("qkv"):
        along = draw(rng, x[n].shape, dtype)
        ends, exact, noise = [], [], 0.0
        for sign in (1, -1):
            y = dict(x, **{n: (x[n] + np.float32(sign * h) * along).astype(np.float32)})
            ends.append((y[n].astype(np.float64), host(forward(gpu, on_gpu(gpu, name, y))[0])[:t]))
            ref = O.packed_attention(y["q"], y["k"], y["v"], y["cu"], d ** -0.5, window, sinks)
            exact.append(ref[0][:t])
            noise += (tolerances(name, ref)[0][:t] * np.abs(x["do"][:t])).sum() / (2 * h)
        quotient = ((ends[0][1] - ends[1][1]) * x["do"][:t]).sum() / (2 * h)
        true = ((exact[0] - exact[1]) * x["do"][:t]).sum() / (2 * h)
        step = ((ends[0][0] - ends[1][0]) / (2 * h))[:t]
        ref = O.packed_attention(x["q"], x["k"], x["v"], x["cu"], d ** -0.5, window, sinks)
        of_out, _, of_weight = tolerances(name, ref)
        sums = (max(lens) * (hq // hk) + 64) * E
        grads, bounds = O.packed_attention_backward(x["q"], x["k"], x["v"], x["do"], x["cu"], d ** -0.5, window, sinks, of_out,
                                                    of_weight + sums, 0.0, (d + 10) * E + sums)
        tol = noise + abs(true - (grads[i][:t] * step).sum()) + ((E * np.abs(grads[i]) + 2 * bounds[i])[:t] * np.abs(step)).sum()
        assert abs(quotient - (got[i][:t] * step).sum()) <= tol, (name, n, quotient, (got[i][:t] * step).sum(), tol)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("window", [0, 50])
def test_other_sequences_and_the_space_behind(gpu, dtype, window):
    """Infinities and NaNs in other sequences' rows and behind the last one
    reach nothing."""
    import torch
    lens = [70, 45, 133]
    cu = torch.tensor([0, 70, 115, 248], dtype=torch.int32, device="cuda")
    cfg = gpu.heads_config(4, 2, 64, dtype=dtype, norm=False, rot_dim=0)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    torch.manual_seed(5)
    q, do = (torch.randn(260, 4, 64, device="cuda").to(dt) for _ in range(2))
    k, v = (torch.randn(260, 2, 64, device="cuda").to(dt) for _ in range(2))

    def both():
        out, lse = gpu.packed_attention_forward(cfg, q, k, v, cu, 133, window=window, sinks=3)
        return out, lse, *gpu.packed_attention_backward(cfg, q, k, v, out, lse, do, cu, 133, window=window, sinks=3)

    clean = both()
    for x in (q, k, v, do):
        x[70:115] = float("nan")
        x[90:100] = float("inf")
        x[248:] = float("nan")
    for a, b in zip(clean, both()):
        assert torch.equal(a[:70], b[:70]) and torch.equal(a[115:248], b[115:248])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_what_windows_leave_behind(gpu, dtype, d):
    """Infinities and NaNs in rows that windows of 50 have left reach neither
    results nor gradients of tokens 128 (a workgroup's) and more past the last
    that sees them, first rows in sight or not; nor, on the way back, those of
    tokens 128 and more before them."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    cfg = gpu.heads_config(4, 2, d, dtype=dtype, norm=False, rot_dim=0)
    cu = torch.tensor([0, 700], dtype=torch.int32, device="cuda")
    torch.manual_seed(6)
    x = [torch.randn(700, h, d, device="cuda").to(dt) for h in (4, 2, 2, 4)]
    for sinks in (0, 3):
        def both():
            q, k, v, do = x
            out, lse = gpu.packed_attention_forward(cfg, q, k, v, cu, 700, window=50, sinks=sinks)
            return out, *gpu.packed_attention_backward(cfg, q, k, v, out, lse, do, cu, 700, window=50, sinks=sinks)

        clean = both()
        keep = [y.clone() for y in x]
        for y in x:
            y[300:310] = float("nan")
            y[305] = float("inf")
        got = both()
        for y, z in zip(x, keep):
            y.copy_(z)
        for i, (a, b) in enumerate(zip(clean, got)):
            assert torch.equal(a[310 + 49 + 128:], b[310 + 49 + 128:]), (sinks, i)
            first = 128 if sinks and i > 1 else 0  # (the first rows' keys are seen by the spoilt queries)
            assert torch.equal(a[first:300 - 128], b[first:300 - 128]), (sinks, i)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_bands_of_one_buffer_and_rows_far_apart(gpu, dtype):
    """dq, dk and dv as bands of one buffer; tokens 2^24 bytes apart."""
    import torch
    x = inputs("group_of_5" if dtype == "bf16" else "long_fp32", 6)
    name = "group_of_5" if dtype == "bf16" else "long_fp32"
    g = on_gpu(gpu, name, x)
    out, lse = forward(gpu, g)
    plain = backward(gpu, g, out, lse)
    lens, hq, hk, d, *_ = CASES[name]
    t = sum(lens)
    wide = torch.full((t, hq + 2 * hk + 1, d), 7.0, dtype=out.dtype, device="cuda")
    bands = wide[:, :hq], wide[:, hq:hq + hk], wide[:, hq + hk + 1:]
    backward(gpu, g, out, lse, dq=bands[0], dk=bands[1], dv=bands[2])
    assert all(torch.equal(a, b) for a, b in zip(plain, bands)) and (wide[:, hq + hk] == 7).all()
    # few tokens whose rows lie 16 MB apart
    es = out.element_size()
    cu = torch.tensor([0, 20, 33], dtype=torch.int32, device="cuda")
    far = {}
    for n, h in (("q", hq), ("k", hk), ("v", hk), ("do", hq)):
        room = torch.empty(33 * (1 << 24) // es, dtype=out.dtype, device="cuda")
        far[n] = room.as_strided((33, h, d), ((1 << 24) // es, d, 1))
        far[n].copy_(g[n][:33])
    near = {n: far[n].contiguous() for n in far}
    got = []
    for s in (near, far):
        o, l = gpu.packed_attention_forward(g["cfg"], s["q"], s["k"], s["v"], cu, 20)
        got.append((o, l, *gpu.packed_attention_backward(g["cfg"], s["q"], s["k"], s["v"], o, l, s["do"], cu, 20)))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_sequences(gpu, dtype):
    """3,000 sequences of up to five tokens, each against itself alone."""
    import torch
    rng = np.random.default_rng(7)
    lens = rng.integers(0, 6, 3000)
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).cuda()
    t = int(cu[-1])
    cfg = gpu.heads_config(4, 2, 64, dtype=dtype, norm=False, rot_dim=0)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q, do = (torch.randn(t, 4, 64, device="cuda").to(dt) for _ in range(2))
    k, v = (torch.randn(t, 2, 64, device="cuda").to(dt) for _ in range(2))
    out, lse = gpu.packed_attention_forward(cfg, q, k, v, cu, 5)
    got = gpu.packed_attention_backward(cfg, q, k, v, out, lse, do, cu, 5)
    for s in rng.integers(0, 3000, 40):
        a, b = int(cu[s]), int(cu[s + 1])
        if a == b:
            continue
        one = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
        o, l = gpu.packed_attention_forward(cfg, q[a:b], k[a:b], v[a:b], one, 5)
        alone = gpu.packed_attention_backward(cfg, q[a:b], k[a:b], v[a:b], o, l, do[a:b], one, 5)
        for x, y in zip((o, l, *alone), (out, lse, *got)):
            assert torch.equal(x, y[a:b])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_past_32_bits(gpu, dtype):
    """The inputs' and gradients' rows 2^24 bytes apart, more than 4 GiB each
    (out and lse are dense)."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    d, lens = 64, (130, 0, 150)
    t = sum(lens)
    cfg = gpu.heads_config(2, 1, d, dtype=dtype, norm=False, rot_dim=0)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    step = (1 << 24) // dt.itemsize

    def far(h):
        return torch.empty((t - 1) * step + h * d, dtype=dt, device="cuda").as_strided((t, h, d), (step, d, 1))

    near = {n: torch.randn(t, h, d, device="cuda").to(dt) for n, h in (("q", 2), ("k", 1), ("v", 1), ("do", 2))}
    apart = {n: far(x.shape[1]).copy_(x) for n, x in near.items()}
    out, lse = gpu.packed_attention_forward(cfg, near["q"], near["k"], near["v"], cu, 150)
    want = out, lse, *gpu.packed_attention_backward(cfg, near["q"], near["k"], near["v"], out, lse, near["do"], cu, 150)
    o, l = gpu.packed_attention_forward(cfg, apart["q"], apart["k"], apart["v"], cu, 150)
    got = o, l, *gpu.packed_attention_backward(cfg, apart["q"], apart["k"], apart["v"], o, l, apart["do"], cu, 150, dq=far(2),
                                               dk=far(1), dv=far(1))
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_tokens_past_32_bits(gpu):
    """90,000 sequences whose tensors hold more than 4 GiB each: those around
    2 and 4 GiB and the last against themselves alone."""
    import torch
    lens = np.random.default_rng(13).integers(0, 201, 90000)
    ends = np.concatenate([[0], np.cumsum(lens)])
    cu = torch.from_numpy(ends.astype(np.int32)).cuda()
    t, d = int(ends[-1]), 64
    assert t * 4 * d * 2 > 1 << 32
    cfg = gpu.heads_config(4, 4, d, norm=False, rot_dim=0)
    q, k, v, do = (torch.randn(t, 4, d, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    out, lse = gpu.packed_attention_forward(cfg, q, k, v, cu, 200)
    got = gpu.packed_attention_backward(cfg, q, k, v, out, lse, do, cu, 200)
    seqs = [int(np.searchsorted(ends, n // (4 * d * 2), "right")) - 1 + i for n in (1 << 31, 1 << 32) for i in range(-2, 3)]
    for s in seqs + [0, 89997, 89998, 89999]:
        a, b = int(ends[s]), int(ends[s + 1])
        if a == b:
            continue
        one = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
        o, l = gpu.packed_attention_forward(cfg, q[a:b], k[a:b], v[a:b], one, 200)
        alone = gpu.packed_attention_backward(cfg, q[a:b], k[a:b], v[a:b], o, l, do[a:b], one, 200)
        for x, y in zip((o, l, *alone), (out, lse, *got)):
            assert torch.equal(x, y[a:b]), s


def test_max_len_lays_out_only(gpu):
    """A launch laid out for fewer or more tokens than there are is right too."""
    import torch
    name = "workgroup_edges"
    x = inputs(name, 8)
    g = on_gpu(gpu, name, x)
    ref = O.packed_attention(x["q"], x["k"], x["v"], x["cu"], 128 ** -0.5)
    t = x["cu"][-1]
    for most in (1, 100000):
        g["most"] = most
        out, lse = forward(gpu, g)
        close(host(out)[:t], ref[0][:t], tolerances(name, ref)[0][:t], most)
        check_backward(name, x, backward(gpu, g, out, lse), ref, 128 ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_in_a_graph_and_on_another_stream(gpu, dtype):
    """Both directions captured and replayed on new inputs and lengths, eager
    calls of the same buffers between replays."""
    import torch
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    cfg = gpu.heads_config(6, 2, 64, dtype=dtype, norm=False, rot_dim=0)
    q, do = (torch.randn(300, 6, 64, device="cuda").to(dt) for _ in range(2))
    k, v = (torch.randn(300, 2, 64, device="cuda").to(dt) for _ in range(2))
    cu = torch.tensor([0, 100, 290], dtype=torch.int32, device="cuda")
    ws = torch.empty(gpu.load().proxy_packed_workspace_size(cfg, 2, 300, 300, 90, 2), dtype=torch.uint8, device="cuda")

    def both(ws=None, stream=None):
        out, lse = gpu.packed_attention_forward(cfg, q, k, v, cu, 300, window=90, sinks=2, stream=stream)
        return out, lse, *gpu.packed_attention_backward(cfg, q, k, v, out, lse, do, cu, 300, window=90, sinks=2, workspace=ws,
                                                        stream=stream)

    both(ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(ws)
    for i, ends in enumerate(([0, 100, 290], [0, 0, 300], [0, 299, 300], [0, 1, 2])):
        for x in (q, k, v, do):
            x.copy_(torch.randn_like(x))
        cu.copy_(torch.tensor(ends, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        seen = [x[:ends[-1]].clone() for x in got]
        for x, y in zip(seen, both()):
            assert torch.equal(x, y[:ends[-1]])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = both(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(other, both()):
        assert torch.equal(x[:2], y[:2])


def test_norm_rotation_attention_and_back(gpu):
    """A training step of the layer's attention: norm and rotation, attention,
    and both backwards, against automatic differentiation in 64 bits. In fp32:
    each gradient within 2^-16 of the terms' size, sums of 120 rows of 64
    channels chained twice (a few hundred roundings of 2^-24)."""
    import torch
    torch.manual_seed(9)
    t, hq, hk, d = 120, 4, 2, 64
    cfg = gpu.heads_config(hq, hk, d, dtype="fp32", eps=1e-5)
    freqs = gpu.rope_freqs(cfg)
    w = {"gamma_q": 1 + 0.1 * torch.randn(d, device="cuda"), "gamma_k": 1 + 0.1 * torch.randn(d, device="cuda"), "freqs": freqs}
    qkv = torch.randn(t, hq + 2 * hk, d, device="cuda")
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    do = torch.randn(t, hq, d, device="cuda")
    cu = torch.tensor([0, 50, 120], dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(50), torch.arange(70)]).to(torch.int32).cuda()
    qr, kr = gpu.qk_norm_rope_forward(cfg, w, q, k, pos)
    out, lse = gpu.packed_attention_forward(cfg, qr, kr, v, cu, 70)
    dqr, dkr, dv = gpu.packed_attention_backward(cfg, qr, kr, v, out, lse, do, cu, 70)
    dq, dk, dgq, dgk = gpu.qk_norm_rope_backward(cfg, w, q, k, pos, dqr, dkr)

    leaves = [x.detach().cpu().double().requires_grad_() for x in (q, k, v, w["gamma_q"], w["gamma_k"])]
    angle = pos.cpu().double()[:, None] * freqs.cpu()
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]

    def turned(x, g):
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-5) * g
        a, b = x.chunk(2, -1)
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)

    a, b, c = turned(leaves[0], leaves[3]), turned(leaves[1], leaves[4]), leaves[2]
    parts = []
    for lo, hi in ((0, 50), (50, 120)):
        s = torch.einsum("ihd,jhd->hij", a[lo:hi], b[lo:hi].repeat_interleave(hq // hk, 1)) * d ** -0.5
        s = s.masked_fill(torch.ones(hi - lo, hi - lo).triu(1).bool(), float("-inf"))
        parts.append(torch.einsum("hij,jhd->ihd", s.softmax(-1), c[lo:hi].repeat_interleave(hq // hk, 1)))
    want = torch.autograd.grad(torch.cat(parts), leaves, do.cpu().double())
    for x, y in zip((dq, dk, dv, dgq, dgk), want):
        assert (x.cpu().double() - y).abs().max() <= 2.0 ** -16 * y.abs().max()


def test_no_tokens(gpu):
    import torch
    cfg = gpu.heads_config(4, 2, 64, norm=False, rot_dim=0)
    e = lambda h: torch.empty(0, h, 64, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    cu = torch.zeros(3, dtype=torch.int32, device="cuda")
    out, lse = gpu.packed_attention_forward(cfg, e(4), e(2), e(2), cu, 1)
    dq, dk, dv = gpu.packed_attention_backward(cfg, e(4), e(2), e(2), out, lse, e(4), cu, 1)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4) and dk.shape == (0, 2, 64)


def test_the_binding_refuses(gpu):
    import torch
    cfg = gpu.heads_config(4, 2, 64, norm=False, rot_dim=0)
    r = lambda h, dt=torch.bfloat16, d="cuda": torch.zeros(9, h, 64, dtype=dt, device=d)  # noqa: E731
    cu = torch.tensor([0, 9], dtype=torch.int32, device="cuda")
    for bad in (dict(q=r(5)), dict(k=r(4)), dict(v=r(2, torch.float32)), dict(cu=cu.long()), dict(cu=cu.cpu()), dict(q=r(4, d="cpu")),
                dict(cu=cu[None]), dict(v=r(2).transpose(1, 2).contiguous().transpose(1, 2))):
        a = dict(q=r(4), k=r(2), v=r(2), cu=cu)
        a.update(bad)
        with pytest.raises(ValueError):
            gpu.packed_attention_forward(cfg, a["q"], a["k"], a["v"], a["cu"], 9)
    for kw in (dict(out=r(2)), dict(out=r(4).float()), dict(lse=torch.zeros(9, 4, device="cuda").double())):
        with pytest.raises(ValueError):
            gpu.packed_attention_forward(cfg, r(4), r(2), r(2), cu, 9, **kw)
    out, lse = gpu.packed_attention_forward(cfg, r(4), r(2), r(2), cu, 9)
    for kw in (dict(dq=r(2)), dict(dk=r(4)), dict(workspace=torch.zeros(9, device="cpu"))):
        with pytest.raises(ValueError):
            gpu.packed_attention_backward(cfg, r(4), r(2), r(2), out, lse, r(4), cu, 9, **kw)
    with pytest.raises(gpu.ProxyFormerError):
        gpu.packed_attention_backward(cfg, r(4), r(2), r(2), out, lse, r(4), cu, 9, workspace=torch.zeros(16, device="cuda"))
