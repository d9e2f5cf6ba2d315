"""The fine tokens' own attention on the GPU against the float64 oracle: norm
and rotation (forward, backward), append into a paged cache and attention over
it, alone and as they are used together.

Tolerances, per element, from the roundings that can occur (u: half a step of
the result's type, 2^-8 of it in bf16 and 2^-24 in fp32; E = 2^-24):
* norm and rotation: u |y| + 32 E m. m is what the rotation can carry into the
  element. 128 squares are summed in chains of 16 and a tree of 3 (halved by
  the root: 10 E), root, gain and product 4 E, the angle 2 E (below half a
  revolution in fp32), cosine and sine 4 E, the turn 4 E.
* its gradient: u |dx| + 64 E m: the same twice, and a mean of 128 products.
* gains' gradients: 128 E m, m the sum of the terms' magnitudes: the terms 40 E
  and sums along at most 64 additions.
* attention: u |o| + (2 d + (n + 64) E + r) m, m = sum p |v|, n rows seen.
  d, a score's error: (D + 10) E s + 8 E, s the largest sum of |q||k| terms
  times the scale; the weights' errors enter once above and once below the
  fraction. r = 2^-17 in bf16, whose weights enter as two terms; 2^-8 where a
  prompt of 32 or more tokens is laid out for, whose weights enter as one
  (their sum is taken before that rounding).
* lse: 2 d + (n + 64) E + 4 E |lse|.
"""
import numpy as np
import pytest

from oracle import heads as O
from paper_2608_23463_amd import synth
from helpers import dev, host, torch_dtype

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {"bf16": 2.0 ** -8, "fp32": E}


def draw(rng, shape, dtype, scale=1.0):
    a = (rng.standard_normal(shape) * scale).astype(np.float32)
    return synth.bf16_round(a) if dtype == "bf16" else a


def close(got, ref, tol, what):
    got = np.asarray(got)
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (what, int(bad.sum()), got.size, got[bad][:4], ref[bad][:4], np.broadcast_to(tol, ref.shape)[bad][:4])


def laid_out(a, dtype, layout, extra=2):
    """A tensor [T, H, D] of the values a: contiguous, a band of a wider buffer, or heads first."""
    import torch
    t = dev(a, dtype)
    if layout == "band":
        wide = torch.full((t.shape[0], t.shape[1] + extra, t.shape[2]), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, 1:1 + t.shape[1]] = t
        return wide[:, 1:1 + t.shape[1]]
    if layout == "heads":
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    return t


CASES = {
    # name: (tokens, heads, kv heads, head_dim, dtype, norm, rot, pairs style, axes, layout)
    "T1_h16x64": (1, 16, 16, 64, "bf16", True, 64, False, (32,), "plain"),
    "T3_h1x128_fp32_pairs": (3, 1, 1, 128, "fp32", True, 128, True, (64,), "plain"),
    "T5_h5_1x64_band": (5, 5, 1, 64, "bf16", True, 32, False, (16,), "band"),
    "T67_h12_4x128_video": (67, 12, 4, 128, "bf16", True, 96, False, (16, 16, 16), "heads"),
    "T130_h17x64_fp32_uneven_axes": (130, 17, 17, 64, "fp32", True, 48, True, (1, 23), "band"),
    "T33_no_norm": (33, 8, 2, 64, "bf16", False, 64, True, (32,), "heads"),
    "T33_norm_only": (33, 8, 2, 128, "fp32", True, 0, False, (0,), "plain"),
    "T9_neither": (9, 4, 4, 64, "bf16", False, 0, False, (0,), "band"),
    "T2049_h3x128_rot16": (2049, 3, 3, 128, "bf16", True, 16, True, (8,), "plain"),
    "T4099_h8_2x64_fp32": (4099, 8, 2, 64, "fp32", True, 64, False, (32,), "band"),
    "T5000_h9_3x64": (5000, 9, 3, 64, "bf16", True, 64, False, (20, 12), "heads"),
}


def qk_inputs(B, case, seed):
    t, hq, hk, d, dtype, norm, rot, pairs, axes, layout = case
    rng = np.random.default_rng(seed)
    cfg = B.heads_config(hq, hk, d, dtype=dtype, norm=norm, eps=1e-5, rot_dim=rot,
                         style=B.PF_ROPE_PAIRS if pairs else B.PF_ROPE_HALVES, axis_pairs=axes)
    freqs = B.rope_freqs(cfg)
    pos = rng.integers(0, 1 << 20, (len(axes), t)).astype(np.int32)
    pos[0, 0] = -7
    g = [draw(rng, d, dtype) * 0.25 + 1 if norm else None for _ in range(2)]
    if norm and dtype == "bf16":
        g = [synth.bf16_round(x.astype(np.float32)) for x in g]
    import torch
    a = {"cfg": cfg, "ang": O.angles(pos, host64(freqs), axes), "pos": torch.from_numpy(pos).cuda(),
         "q": draw(rng, (t, hq, d), dtype, 3), "k": draw(rng, (t, hk, d), dtype, 0.1),
         "dq": draw(rng, (t, hq, d), dtype), "dk": draw(rng, (t, hk, d), dtype), "g": g,
         "w": {"gamma_q": dev(g[0], dtype), "gamma_k": dev(g[1], dtype), "freqs": freqs}}
    return a


def host64(t):
    return t.detach().cpu().double().numpy()


@pytest.mark.parametrize("name", CASES)
def test_forward(gpu, name):
    import torch
    B, case = gpu, CASES[name]
    t, hq, hk, d, dtype, norm, rot, pairs, axes, layout = case
    a = qk_inputs(B, case, 1)
    q, k = laid_out(a["q"], dtype, layout), laid_out(a["k"], dtype, layout)
    qo, ko = B.qk_norm_rope_forward(a["cfg"], a["w"], q, k, a["pos"])
    qi, ki = q.clone(memory_format=torch.preserve_format), k.clone(memory_format=torch.preserve_format)
    B.qk_norm_rope_forward(a["cfg"], a["w"], qi, ki, a["pos"], qi, ki)  # in place
    torch.cuda.synchronize()
    assert torch.equal(qi, qo) and torch.equal(ki, ko)
    for got, x, g in ((qo, a["q"], a["g"][0]), (ko, a["k"], a["g"][1])):
        ref, mag = O.norm_rope(x, g, 1e-5, norm, a["ang"], rot, pairs)
        close(host(got), ref, U[dtype] * np.abs(ref) + 32 * E * mag, name)


@pytest.mark.parametrize("name", CASES)
def test_backward(gpu, name):
    import torch
    B, case = gpu, CASES[name]
    t, hq, hk, d, dtype, norm, rot, pairs, axes, layout = case
    a = qk_inputs(B, case, 2)
    q, k = laid_out(a["q"], dtype, layout), laid_out(a["k"], dtype, layout)
    dqo, dko = laid_out(a["dq"], dtype, layout), laid_out(a["dk"], dtype, layout)
    got = B.qk_norm_rope_backward(a["cfg"], a["w"], q, k, a["pos"], dqo, dko)
    again = B.qk_norm_rope_backward(a["cfg"], a["w"], q, k, a["pos"], dqo, dko, dq=dqo, dk=dko)  # in place
    torch.cuda.synchronize()
    for x, y in zip(got, again):
        assert (x is None and y is None) or torch.equal(x, y)
    for i, (x, g, dy) in enumerate(((a["q"], a["g"][0], a["dq"]), (a["k"], a["g"][1], a["dk"]))):
        dx, dg, mag, dg_mag = O.norm_rope_backward(x, g, 1e-5, norm, a["ang"], rot, pairs, dy)
        close(host(got[i]), dx, U[dtype] * np.abs(dx) + 64 * E * mag, (name, i))
        if norm:
            close(host(got[2 + i]), dg, 128 * E * dg_mag, (name, "gain", i))
        else:
            assert got[2 + i] is None


@pytest.mark.parametrize("name", ["T3_h1x128_fp32_pairs", "T130_h17x64_fp32_uneven_axes", "T33_norm_only"])
def test_backward_against_differences(gpu, name):
    """The backward's derivative along a direction against a central difference
    of the forward's results. The difference's own error is its distance in
    float64 (the oracle's difference against its derivative) and the forward's
    roundings (33 E m per element, twice) over the step."""
    import torch
    B, case = gpu, CASES[name]
    t, hq, hk, d, dtype, norm, rot, pairs, axes, layout = case
    a = qk_inputs(B, case, 3)
    rng = np.random.default_rng(4)
    h = 2.0 ** -7
    along = {x: draw(rng, a[x].shape, dtype, float(np.abs(a[x]).mean())) for x in ("q", "k")}
    dq, dk, _, _ = B.qk_norm_rope_backward(a["cfg"], a["w"], dev(a["q"], dtype), dev(a["k"], dtype), a["pos"],
                                           dev(a["dq"], dtype), dev(a["dk"], dtype))
    ends = []
    for sign in (1, -1):
        at = [(a[x] + np.float32(sign * h) * along[x]).astype(np.float32) for x in ("q", "k")]
        out = B.qk_norm_rope_forward(a["cfg"], a["w"], dev(at[0], dtype), dev(at[1], dtype), a["pos"])
        torch.cuda.synchronize()
        ends.append([(at[i].astype(np.float64), host(out[i])) for i in range(2)])
    for i, (x, dy, got) in enumerate((("q", a["dq"], host(dq)), ("k", a["dk"], host(dk)))):
        g = a["g"][i]
        exact = [O.norm_rope(e[i][0], g, 1e-5, norm, a["ang"], rot, pairs) for e in ends]
        quotient = ((ends[0][i][1] - ends[1][i][1]) * dy).sum() / (2 * h)
        ref = ((exact[0][0] - exact[1][0]) * dy).sum() / (2 * h)
        step = (ends[0][i][0] - ends[1][i][0]) / (2 * h)  # the direction as fp32 took it
        dx, _, mag, _ = O.norm_rope_backward(a[x], g, 1e-5, norm, a["ang"], rot, pairs, dy)
        noise = sum((33 * E * e[1] * np.abs(dy)).sum() for e in exact) / (2 * h)
        tol = noise + abs(ref - (dx * step).sum()) + ((E * np.abs(dx) + 64 * E * mag) * np.abs(step)).sum()
        assert abs(quotient - (got * step).sum()) <= tol, (name, x, quotient, (got * step).sum(), tol)
        assert tol < 0.05 * np.sqrt((dx ** 2).sum() * (step ** 2).sum())  # the comparison says something


def test_training_calls_in_a_graph(gpu):
    """Forward and backward captured together and replayed on new inputs, an
    eager call of the same buffers between replays."""
    import torch
    B, case = gpu, CASES["T67_h12_4x128_video"]
    a = qk_inputs(B, case, 5)
    dt = case[4]
    q, k, dq, dk = (dev(a[x], dt) for x in ("q", "k", "dq", "dk"))

    def both():
        out = B.qk_norm_rope_forward(a["cfg"], a["w"], q, k, a["pos"])
        return (*out, *B.qk_norm_rope_backward(a["cfg"], a["w"], q, k, a["pos"], dq, dk))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for i in range(4):
        for x in (q, k, dq, dk):
            x.copy_(torch.randn_like(x))
        graph.replay()
        torch.cuda.synchronize()
        seen = [x.clone() for x in got]
        for x, y in zip(seen, both()):
            assert torch.equal(x, y)


def test_no_tokens_and_missing_gains(gpu):
    import torch
    B = gpu
    cfg = B.heads_config(4, 2, 64, dtype="fp32")
    w = {"freqs": B.rope_freqs(cfg)}
    z = lambda n, h: torch.randn(n, h, 64, device="cuda")  # noqa: E731
    pos = torch.zeros(1, 0, dtype=torch.int32, device="cuda")
    dq, dk, gq, gk = B.qk_norm_rope_backward(cfg, w, z(0, 4), z(0, 2), pos, z(0, 4), z(0, 2))
    torch.cuda.synchronize()
    assert dq.shape == (0, 4, 64) and (gq == 0).all() and (gk == 0).all()
    q, k, pos = z(7, 4), z(7, 2), torch.arange(7, dtype=torch.int32, device="cuda")
    ones = dict(w, gamma_q=torch.ones(64, device="cuda"), gamma_k=torch.ones(64, device="cuda"))
    for a, b in zip(B.qk_norm_rope_forward(cfg, w, q, k, pos), B.qk_norm_rope_forward(cfg, ones, q, k, pos)):
        assert torch.equal(a, b)


# ---------------------------------------------------------------- paged cache

class Paged:
    """A cache whose pages start as NaN; sequences' rows below `filled` hold values."""

    def __init__(self, B, rng, hq, hk, d, dtype, page, lens, filled, norm=False, rot=0, pairs=False, spare=2, extra_pages=1):
        import torch
        self.page, self.lens, self.dtype = page, lens, dtype
        self.cfg = B.heads_config(hq, hk, d, dtype=dtype, norm=norm, rot_dim=rot,
                                  style=B.PF_ROPE_PAIRS if pairs else B.PF_ROPE_HALVES)
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), max(need + [1]) + extra_pages), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, hk, page, d)
        self.k, self.v = np.full(shape, np.nan, np.float32), np.full(shape, np.nan, np.float32)
        for b, n in enumerate(filled):
            for j in range(n):
                pg = self.table[b, j // page]
                self.k[pg, :, j % page] = draw(rng, (hk, d), dtype)
                self.v[pg, :, j % page] = draw(rng, (hk, d), dtype)
        gam = [draw(rng, d, dtype) if norm else None for _ in range(2)]
        self.gammas = gam
        self.weights = {"gamma_q": dev(gam[0], dtype), "gamma_k": dev(gam[1], dtype), "freqs": B.rope_freqs(self.cfg)}
        self.kd, self.vd = dev(self.k, dtype), dev(self.v, dtype)
        self.td = torch.from_numpy(self.table).cuda()
        self.ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.cache = B.PagedCache(self.cfg, self.weights, self.kd, self.vd, self.td, self.ld)


def check_attend(p, q, out, lse, cu, window, sinks, scale, what, max_new=1):
    d, dtype = q.shape[2], p.dtype
    ref, rlse, s, mag = O.paged_attention(q, p.k, p.v, p.table, p.lens, cu, scale, window, sinks)
    n = ref.shape[0] if cu is None else int(cu[-1])
    seen = max([1] + [O.visible(r, max(r + 1, 0), window, sinks).sum() for _, r in O.token_rows(p.lens, cu)])
    dl = ((d + 10) * s + 8) * E
    r = 0.0 if dtype == "fp32" else 2.0 ** -17 if cu is None or max_new < 32 else 2.0 ** -8
    tol = U[dtype] * np.abs(ref) + (2 * dl + (seen + 64) * E + r)[..., None] * mag
    close(host(out)[:n], ref[:n], tol[:n], what)
    if lse is not None:
        got = host(lse)[:n]
        empty = np.isneginf(rlse[:n])
        assert (np.isneginf(got) == empty).all(), what
        close(got[~empty], rlse[:n][~empty], (2 * dl + (seen + 64) * E + 4 * E * np.abs(rlse))[:n][~empty], (what, "lse"))


ONE = {
    # name: (heads, kv heads, head_dim, dtype, page, lengths, window, sinks)
    "B1_n1": (1, 1, 64, "bf16", 16, [1], 0, 0),
    "edges_of_blocks": (4, 2, 128, "bf16", 16, [0, 1, 15, 16, 17, 31, 32, 33, 128, 129], 0, 0),
    "edges_of_blocks_fp32": (4, 2, 64, "fp32", 32, [0, 1, 15, 16, 17, 31, 32, 33, 128, 129], 0, 0),
    "pages_of_48_group3": (6, 2, 64, "bf16", 48, [700, 5, 47, 48, 49, 300], 0, 0),
    "group16": (16, 1, 128, "bf16", 64, [333, 0, 64], 0, 0),
    "group17_fp32_128": (17, 1, 128, "fp32", 16, [200, 77], 0, 0),
    "group40": (80, 2, 64, "bf16", 128, [500, 129], 0, 0),
    "window_1": (2, 2, 64, "bf16", 16, [100, 1, 16], 1, 0),
    "window_33_sinks_5": (8, 2, 128, "bf16", 16, [600, 33, 34, 38, 39, 70], 33, 5),
    "window_100_sinks_70": (4, 4, 64, "fp32", 32, [400, 169, 170, 171, 60], 100, 70),
    "window_past_all": (4, 4, 64, "bf16", 16, [50, 90], 1 << 40, 3),
    "long_and_short": (6, 2, 128, "bf16", 32, [5000, 3, 0, 2100, 700, 0, 1025, 64], 0, 0),
    "long_and_short_mha": (3, 3, 64, "bf16", 16, [0, 2000, 1, 4100, 513], 0, 0),
    "long_and_short_fp32_window": (20, 1, 64, "fp32", 64, [3000, 900, 0, 2000], 1500, 40),
    "many_slots": (2, 1, 64, "bf16", 16, [(37 * i) % 90 for i in range(150)], 0, 0),
}


@pytest.mark.parametrize("name", ONE)
def test_attend_one_token(gpu, name):
    import torch
    hq, hk, d, dtype, page, lens, window, sinks = ONE[name]
    rng = np.random.default_rng(5)
    p = Paged(gpu, rng, hq, hk, d, dtype, page, lens, lens)
    # rows out of sight hold NaN and infinities
    if window:
        for b, n in enumerate(lens):
            for j in np.nonzero(~O.visible(n - 1, max(n, 0), window, sinks))[0]:
                pg = p.table[b, j // page]
                p.k[pg, :, j % page] = np.nan
                p.v[pg, :, j % page] = np.inf if j % 2 else np.nan
        p.kd.copy_(dev(p.k, dtype))
        p.vd.copy_(dev(p.v, dtype))
    q = draw(rng, (len(lens), hq, d), dtype, 2)
    scale = 0.7 / np.sqrt(d)
    outs = []
    for hint in (max(lens + [1]), 1, 5000):  # the length the launch is laid out for does not matter
        lse = torch.full((len(lens), hq), float("nan"), device="cuda")
        out = p.cache.attend(laid_out(q, dtype, "band"), hint, window=window, sinks=sinks, scale=scale, lse=lse)
        torch.cuda.synchronize()
        check_attend(p, q, out, lse, None, window, sinks, scale, (name, hint))
        outs.append(out)
    again = p.cache.attend(laid_out(q, dtype, "band"), max(lens + [1]), window=window, sinks=sinks, scale=scale)
    assert torch.equal(again, outs[0])


PROMPTS = {
    # name: (heads, kv heads, head_dim, dtype, page, lengths, new tokens, padding, window, sinks)
    "one_of_1": (2, 1, 64, "bf16", 16, [1], [1], 0, 0, 0),
    "from_the_start": (4, 1, 64, "bf16", 16, [70, 33], [70, 33], 3, 0, 0),
    "behind_a_cache": (6, 2, 128, "bf16", 48, [300, 17, 64, 0, 200], [5, 17, 0, 0, 64], 5, 0, 0),
    "group5_window": (10, 2, 64, "bf16", 16, [150, 40, 90], [100, 1, 90], 0, 20, 3),
    "group20": (20, 1, 128, "bf16", 32, [66, 9], [30, 9], 2, 0, 0),
    "fp32_window": (4, 4, 64, "fp32", 32, [130, 64, 65], [129, 2, 64], 1, 50, 60),
    "fp32_128": (3, 3, 128, "fp32", 16, [100, 31], [33, 31], 0, 0, 0),
    "more_new_than_rows": (2, 2, 64, "bf16", 16, [3, 20], [5, 4], 0, 0, 0),
    "long_enough_for_tiles": (4, 2, 64, "bf16", 64, [400, 260, 129], [300, 260, 129], 7, 0, 0),
    "short_behind_a_long_cache": (6, 2, 128, "bf16", 16, [3000, 1500, 40], [40, 33, 0], 0, 0, 0),
    "short_behind_a_long_cache_64": (2, 1, 64, "bf16", 32, [2500, 1025], [5, 35], 2, 1100, 3),
    "long_window_128": (2, 1, 128, "bf16", 16, [390, 200], [257, 200], 0, 70, 4),
}


@pytest.mark.parametrize("name", PROMPTS)
def test_attend_prompts(gpu, name):
    import torch
    hq, hk, d, dtype, page, lens, new, pad, window, sinks = PROMPTS[name]
    rng = np.random.default_rng(6)
    p = Paged(gpu, rng, hq, hk, d, dtype, page, lens, lens)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = int(cu[-1]) + pad
    q = draw(rng, (t, hq, d), dtype, 2)
    scale = 1 / np.sqrt(d)
    for max_new, longest in ((max(new), max(lens)), (1, max(lens)), (4000, 64)):
        out = torch.full((t, hq, d), 7.0, dtype=torch_dtype(dtype), device="cuda")
        lse = torch.full((t, hq), 7.0, device="cuda")
        p.cache.attend(laid_out(q, dtype, "heads"), longest, cu_tokens=torch.from_numpy(cu).cuda(), max_new=max_new,
                       window=window, sinks=sinks, out=out, lse=lse)
        torch.cuda.synchronize()
        check_attend(p, q, out, lse, cu, window, sinks, scale, (name, max_new), max_new)
        assert (out[cu[-1]:] == 7).all() and (lse[cu[-1]:] == 7).all()


def test_thousands_of_sequences(gpu):
    """5,000 sequences in one call, most of them without a new token."""
    import torch
    rng = np.random.default_rng(13)
    nb = 5000
    new = [0] * nb
    for i in (0, 63, 64, 65, 100, 2500, 4095, 4096, 4998):
        new[i] = int(rng.integers(1, 40))
    lens = [n + int(rng.integers(0, 20)) if n else 0 for n in new]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = int(cu[-1]) + 2
    cud = torch.from_numpy(cu).cuda()
    p = Paged(gpu, rng, 2, 1, 64, "bf16", 16, lens, lens)
    q, k = draw(rng, (t, 2, 64), "bf16"), draw(rng, (t, 1, 64), "bf16")
    for max_new in (40, 1):
        out = torch.full((t, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        p.cache.attend(dev(q, "bf16"), max(lens), cu_tokens=cud, max_new=max_new, out=out)
        torch.cuda.synchronize()
        check_attend(p, q, out, None, cu, 0, 0, 64 ** -0.5, max_new, max_new)
        assert (out[-2:] == 7).all()
    p.cache.append(dev(k, "bf16"), dev(k, "bf16"), cu_tokens=cud)
    torch.cuda.synchronize()
    kd = host(p.vd)
    for i, (s, row) in enumerate(O.token_rows(lens, cu)):
        pg, sl = O.place(p.table[s], row, 16, p.n_pages)
        assert np.array_equal(kd[pg, :, sl], k[i])


@pytest.mark.parametrize("past", [50, 700])
@pytest.mark.parametrize("held", [64, 48, 16])
def test_lengths_past_the_table(gpu, held, past):
    """kv_len beyond what the table holds, whether or not that ends a tile: its
    rows are seen, the others are not, and nothing is written past it."""
    import torch
    rng = np.random.default_rng(14)
    p = Paged(gpu, rng, 4, 2, 64, "bf16", 16, [held, 30], [held, 30], extra_pages=0)
    p.lens = [held + past, 30]
    p.ld.copy_(torch.tensor(p.lens, dtype=torch.int32))
    q = draw(rng, (2, 4, 64), "bf16")
    for window, sinks in ((0, 0), (60, 0), (20, 3)):
        out = p.cache.attend(dev(q, "bf16"), 64, window=window, sinks=sinks)
        torch.cuda.synchronize()
        check_attend(p, q, out, None, None, window, sinks, 64 ** -0.5, window)
    before = p.kd.clone()
    kv = dev(draw(rng, (2, 2, 64), "bf16"), "bf16")
    p.cache.append(kv, kv)
    torch.cuda.synchronize()
    assert (p.kd.view(torch.int16) != before.view(torch.int16)).any(-1).any(1).nonzero().tolist() == [[p.table[1, 1], 13]]
    p.lens = [held + past - 30, 30]
    p.ld.copy_(torch.tensor(p.lens, dtype=torch.int32))
    p.kd.copy_(dev(p.k, "bf16"))
    p.vd.copy_(dev(p.v, "bf16"))
    new = np.array([0, 40, 40], np.int32)
    for max_new in (40, 1):
        for window, sinks in ((0, 0), (30, 2)):
            q = draw(rng, (40, 4, 64), "bf16")
            out = p.cache.attend(dev(q, "bf16"), 64, cu_tokens=torch.from_numpy(new).cuda(), max_new=max_new,
                                 window=window, sinks=sinks)
            torch.cuda.synchronize()
            check_attend(p, q, out, None, new, window, sinks, 64 ** -0.5, (max_new, window), max_new)


def test_pages_that_are_none(gpu):
    """Table entries outside the cache: their rows are not seen and not written."""
    import torch
    rng = np.random.default_rng(7)
    for bad in (-1, 10 ** 6, -(1 << 31)):
        p = Paged(gpu, rng, 4, 2, 64, "bf16", 16, [100, 40], [100, 40])
        p.table[0, 2] = p.table[0, 6] = p.table[1, 0] = bad
        p.td.copy_(torch.from_numpy(p.table))
        q = draw(rng, (2, 4, 64), "bf16")
        out = p.cache.attend(dev(q, "bf16"), 100)
        torch.cuda.synchronize()
        check_attend(p, q, out, None, None, 0, 0, 64 ** -0.5, bad)
        before = p.kd.clone(), p.vd.clone()
        kv = dev(draw(rng, (2, 2, 64), "bf16"), "bf16")
        qo = torch.full((2, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        p.cache.append(kv, kv, q=dev(q, "bf16"), q_out=qo)  # row 99 has no page, row 39 has
        torch.cuda.synchronize()
        changed = (p.kd.view(torch.int16) != before[0].view(torch.int16)).any(-1).any(1).nonzero()
        assert changed.tolist() == [[p.table[1, 2], 7]]
        assert (qo[0] == 7).all() and (qo[1] != 7).any()


APPENDS = {
    # name: (heads, kv heads, head_dim, dtype, page, norm, rot, pairs, lengths, new tokens or None, padding)
    "one_each": (8, 2, 64, "bf16", 16, True, 64, False, [1, 16, 17, 300], None, 0),
    "one_each_fp32": (5, 5, 128, "fp32", 48, True, 64, True, [48, 49, 2], None, 0),
    "empty_slots": (4, 2, 64, "bf16", 32, True, 64, False, [0, 33, 0, 1], None, 0),
    "prompts": (6, 2, 128, "bf16", 16, True, 128, False, [70, 5, 40, 0, 33], [70, 0, 17, 0, 33], 9),
    "prompts_fp32_no_norm": (3, 1, 64, "fp32", 64, False, 32, True, [200, 64], [130, 64], 0),
    "many_sequences": (2, 1, 64, "bf16", 16, True, 64, False, [i % 40 for i in range(200)], [i % 40 % 7 for i in range(200)], 3),
    "long": (4, 4, 64, "bf16", 16, True, 64, False, [2500, 1000], [2300, 900], 1),
    "more_new_than_rows": (2, 2, 64, "bf16", 16, True, 64, False, [3, 20], [5, 4], 0),
}


@pytest.mark.parametrize("given", [False, True], ids=["rows", "given_positions"])
@pytest.mark.parametrize("name", APPENDS)
def test_append(gpu, name, given):
    import torch
    hq, hk, d, dtype, page, norm, rot, pairs, lens, new, pad = APPENDS[name]
    rng = np.random.default_rng(8)
    p = Paged(gpu, rng, hq, hk, d, dtype, page, lens, [0] * len(lens), norm=norm, rot=rot, pairs=pairs)
    cu = None if new is None else np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = (len(lens) if new is None else int(cu[-1])) + pad
    q, k, v = draw(rng, (t, hq, d), dtype), draw(rng, (t, hk, d), dtype), draw(rng, (t, hk, d), dtype)
    at = rng.integers(0, 1 << 18, (1, t)).astype(np.int32)
    qo = torch.full((t, hq, d), 7.0, dtype=torch_dtype(dtype), device="cuda")
    p.cache.append(laid_out(k, dtype, "band"), laid_out(v, dtype, "heads"), q=laid_out(q, dtype, "band"), q_out=qo,
                   cu_tokens=None if cu is None else torch.from_numpy(cu).cuda(),
                   positions=torch.from_numpy(at).cuda() if given else None)
    kd, vd = p.kd.clone(), p.vd.clone()
    p.kd.fill_(float("nan"))
    p.cache.append(laid_out(k, dtype, "plain"), laid_out(v, dtype, "plain"),  # without queries
                   cu_tokens=None if cu is None else torch.from_numpy(cu).cuda(),
                   positions=torch.from_numpy(at).cuda() if given else None)
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(p.kd.view(bits), kd.view(bits)) and torch.equal(p.vd.view(bits), vd.view(bits))
    freqs = host64(p.weights["freqs"])
    want_k, tol_k, want_v = p.k.astype(np.float64), np.zeros(p.k.shape), p.v.astype(np.float64)
    want_q, tol_q = np.full(q.shape, 7.0), np.zeros(q.shape)
    first = 0 if cu is None else None
    for i, (s, row) in enumerate(O.token_rows(lens, cu)):
        pl = O.place(p.table[s], row, page, p.n_pages)
        if pl is None:
            continue
        ang = O.angles([[int(at[0, i]) if given else row]], freqs, [rot // 2])
        y, m = O.norm_rope(q[i:i + 1], p.gammas[0], 1e-6, norm, ang, rot, pairs)
        want_q[i], tol_q[i] = y[0], (U[dtype] * np.abs(y) + 32 * E * m)[0]
        y, m = O.norm_rope(k[i:i + 1], p.gammas[1], 1e-6, norm, ang, rot, pairs)
        want_k[pl[0], :, pl[1]], tol_k[pl[0], :, pl[1]] = y[0], (U[dtype] * np.abs(y) + 32 * E * m)[0]
        want_v[pl[0], :, pl[1]] = v[i]
    close(host(qo), want_q, tol_q, name)
    got_k, got_v = host(kd), host(vd)
    assert (np.isnan(got_k) == np.isnan(want_k)).all() and (np.isnan(got_v) == np.isnan(want_v)).all()
    live = ~np.isnan(want_k)
    close(got_k[live], want_k[live], tol_k[live], name)
    assert np.array_equal(got_v[~np.isnan(want_v)], want_v[~np.isnan(want_v)])


@pytest.mark.parametrize("window,sinks", [(24, 2), (0, 0)])
def test_a_conversation_as_it_is_served(gpu, window, sinks):
    """Prompts appended and attended, then steps of one token captured into a
    graph on another stream and replayed while lengths and pages move on; every
    replay against the oracle, with eager calls between them."""
    import torch
    B = gpu
    rng = np.random.default_rng(9)
    hq, hk, d, page, new, steps = 8, 2, 64, 16, [30, 0, 61], 20
    nb = len(new)
    p = Paged(B, rng, hq, hk, d, "bf16", page, [n + steps for n in new], [0] * nb, norm=True, rot=64)
    full = p.table.copy()
    t = sum(new)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    freqs = host64(p.weights["freqs"])

    def appended(q, k, v, rows, qo):
        """What the append should have left; the oracle goes on from the GPU's rounded values."""
        kd, vd, got = host(p.kd), host(p.vd), host(qo)
        for i, (s, row) in enumerate(rows):
            pg, sl = O.place(p.table[s], row, page, p.n_pages)
            ang = O.angles([[row]], freqs, [32])
            for x, g, dst in ((q, p.gammas[0], got[i]), (k, p.gammas[1], kd[pg, :, sl])):
                y, m = O.norm_rope(x[i:i + 1], g, 1e-6, True, ang, 64, False)
                close(dst, y[0], (U["bf16"] * np.abs(y) + 32 * E * m)[0], ("append", i))
            assert np.array_equal(vd[pg, :, sl], v[i])
        p.k, p.v = kd, vd

    q, k, v = (draw(rng, (t, h, d), "bf16") for h in (hq, hk, hk))
    p.lens = list(new)
    p.ld.copy_(torch.tensor(new, dtype=torch.int32))
    cud = torch.from_numpy(cu).cuda()
    qo = p.cache.append(dev(k, "bf16"), dev(v, "bf16"), q=dev(q, "bf16"), cu_tokens=cud)
    out = p.cache.attend(qo, max(new), cu_tokens=cud, max_new=max(new), window=window, sinks=sinks)
    torch.cuda.synchronize()
    appended(q, k, v, O.token_rows(new, cu), qo)
    check_attend(p, host(qo), out, None, cu, window, sinks, d ** -0.5, "prompt", max(new))

    qs, ks, vs = (torch.zeros(nb, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hk))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step(stream=None):
        # the step's lengths grow once, its append and attention both read them
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            p.ld.add_(1)
        qo = p.cache.append(ks, vs, q=qs, stream=stream)
        return qo, p.cache.attend(qo, 600, window=window, sinks=sinks, stream=stream)

    with torch.cuda.stream(side):
        keep = p.ld.clone(), p.kd.clone(), p.vd.clone()
        step()  # warm-up, undone
        p.ld.copy_(keep[0]), p.kd.copy_(keep[1]), p.vd.copy_(keep[2])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        gq, gout = step()
    p.ld.copy_(keep[0])
    for i in range(steps):
        q, k, v = (draw(rng, (nb, h, d), "bf16") for h in (hq, hk, hk))
        for dst, src in ((qs, q), (ks, k), (vs, v)):
            dst.copy_(dev(src, "bf16"))
        if i % 3 == 2:  # an eager step between replays, on a stream of its own
            torch.cuda.synchronize()
            qo, out = step(side)
            side.synchronize()
        else:
            graph.replay()
            qo, out = gq, gout
        torch.cuda.synchronize()
        p.lens = [n + 1 for n in p.lens]
        assert p.ld.tolist() == p.lens
        appended(q, k, v, O.token_rows(p.lens, None), qo)
        check_attend(p, host(qo), out, None, None, window, sinks, d ** -0.5, ("step", i))
    assert np.array_equal(p.td.cpu().numpy(), full)


def test_two_streams_at_once(gpu):
    """Calls on two streams, each with a workspace of its own, give what they give alone."""
    import torch
    rng = np.random.default_rng(10)
    p = Paged(gpu, rng, 4, 1, 128, "bf16", 16, [900, 700], [900, 700])
    qs = [dev(draw(rng, (2, 4, 128), "bf16"), "bf16") for _ in range(2)]
    alone = [p.cache.attend(q, 900).clone() for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        outs = [p.cache.attend(q, 900, stream=s) for q, s in zip(qs, streams)]
        torch.cuda.synchronize()
        for a, b in zip(outs, alone):
            assert torch.equal(a, b)


def test_cache_past_32_bits(gpu):
    """Rows whose byte offsets pass 2^32: the last pages of a 5 GiB pool of keys and of values."""
    import torch
    rng = np.random.default_rng(11)
    hk, d, page = 2, 128, 64
    n_pages = (5 << 30) // (hk * page * d * 2)
    kp = torch.full((n_pages, hk, page, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    vp = torch.full_like(kp, float("nan"))
    table = np.array([[n_pages - 1, 0, n_pages - 3]], np.int32)
    n = 2 * page + 17
    cfg = gpu.heads_config(4, hk, d, norm=False, rot_dim=0)
    cache = gpu.PagedCache(cfg, {}, kp, vp, torch.from_numpy(table).cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    k, v, q = draw(rng, (n, hk, d), "bf16"), draw(rng, (n, hk, d), "bf16"), draw(rng, (1, 4, d), "bf16")
    cache.append(dev(k, "bf16"), dev(v, "bf16"), cu_tokens=torch.tensor([0, n], dtype=torch.int32, device="cuda"))
    out = cache.attend(dev(q, "bf16"), n)
    torch.cuda.synchronize()
    assert torch.equal(kp[n_pages - 3, :, 16].float().cpu(), torch.from_numpy(k[n - 1]).float())
    sc = np.einsum("hd,jhd->hj", q[0].astype(np.float64), np.repeat(k, 2, 1).astype(np.float64)) / np.sqrt(d)
    w = np.exp(sc - sc.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    vv = np.repeat(v, 2, 1).astype(np.float64)
    ref, mag = np.einsum("hj,jhd->hd", w, vv), np.einsum("hj,jhd->hd", w, np.abs(vv))
    s = np.einsum("hd,jhd->hj", np.abs(q[0]), np.abs(np.repeat(k, 2, 1))).max() / np.sqrt(d)
    tol = 2.0 ** -8 * np.abs(ref) + (2 * ((d + 10) * s + 8) * E + (n + 64) * E + 2.0 ** -17) * mag
    close(host(out)[0], ref, tol, "far")


def test_binding_refusals(gpu):
    import torch
    B = gpu
    rng = np.random.default_rng(12)
    p = Paged(B, rng, 4, 2, 64, "bf16", 16, [20, 20], [20, 20])
    q = dev(draw(rng, (2, 4, 64), "bf16"), "bf16")
    kv = dev(draw(rng, (2, 2, 64), "bf16"), "bf16")
    for bad in (lambda: p.cache.attend(q.float(), 20), lambda: p.cache.attend(q[:, :3], 20),
                lambda: p.cache.attend(q.cpu(), 20), lambda: p.cache.attend(q.transpose(1, 2).contiguous().transpose(1, 2), 20),
                lambda: p.cache.attend(q, 20, cu_tokens=torch.zeros(2, dtype=torch.int32, device="cuda")),
                lambda: p.cache.attend(q, 20, out=torch.zeros(2, 4, 128, device="cuda", dtype=torch.bfloat16)[..., :64]),
                lambda: p.cache.attend(q, 20, lse=torch.zeros(2, 4, device="cuda", dtype=torch.bfloat16)),
                lambda: p.cache.append(kv, kv, q_out=q), lambda: p.cache.append(kv, kv[:1]),
                lambda: p.cache.append(kv, kv, positions=torch.zeros(1, 2, dtype=torch.int64, device="cuda")),
                lambda: B.PagedCache(p.cfg, {}, p.kd, p.vd, p.td.long(), p.ld),
                lambda: B.PagedCache(p.cfg, {}, p.kd, p.vd[:1], p.td, p.ld)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: p.cache.attend(q, 0), lambda: p.cache.attend(q, 20, out=q), lambda: p.cache.attend(q[:1], 20),
                lambda: p.cache.attend(q, 5000, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")),
                lambda: p.cache.append(p.kd[:2, :, 0], kv)):
        with pytest.raises(B.ProxyFormerError):
            bad()
