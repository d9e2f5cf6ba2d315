"""The fine tokens' own attention on the GPU where its kernels change course:
references of a softmax that have to be raised, values far from one, sums over
many steps. Oracle and tolerances are those of test_gpu_heads.py."""
import numpy as np
import pytest

from oracle import heads as O
from helpers import dev, host
from test_gpu_heads import E, U, Paged, check_attend, close, draw, laid_out, qk_inputs

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- softmax references

def rising(rng, p, lens, new, hq, d, rise, step):
    """Keys and queries of which every third token's even heads score `rise`
    (units of log2) more at the last rows than at the first 64, in one step or
    row by row, and the others about the same everywhere: u.u = d, q = 2 u, so
    a row a u adds 2 a sqrt(d) log2(e)."""
    u = np.sign(rng.standard_normal(d)).astype(np.float32)
    for b, n in enumerate(lens):
        for j in range(n):
            share = 0.0 if j < 64 else 1.0 if step else (j - 64) / (n - 64)
            pg = p.table[b, j // p.page]
            k = rng.standard_normal((p.k.shape[1], d)) * 0.5 + share * rise / (2 * np.sqrt(d) * np.log2(np.e)) * u
            p.k[pg, :, j % p.page] = np.float32(dev(k.astype(np.float32), "bf16").float().cpu().numpy())
    t = sum(new)
    q = rng.standard_normal((t, hq, d)) * 0.05
    q[1::3, ::2] += 2 * u
    return dev(q.astype(np.float32), "bf16").float().cpu().numpy()


@pytest.mark.parametrize("step", [True, False], ids=["step", "slope"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 3)])
@pytest.mark.parametrize("rise", [20, 60, 250])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_rise(gpu, d, rise, window, sinks, step):
    """Later keys score far above a prompt's first tile, for some columns of a
    wave: sums below, at and past every limit on them, up to exponentials that
    are infinite against the first reference. Whole and cut into slices; values
    of 1 and of 2^70, whose weighted sums stay finite only against a reference
    near the maximum."""
    import torch
    rng = np.random.default_rng(21)
    hq, lens, new = 4, [390, 200], [160, 200]
    p = Paged(gpu, rng, hq, 2, d, "bf16", 16, lens, lens)
    q = rising(rng, p, lens, new, hq, d, rise, step)
    p.kd.copy_(dev(p.k, "bf16"))
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    for size in (1.0, 2.0 ** 70):
        p.v *= np.float32(size)
        p.vd.copy_(dev(p.v, "bf16"))
        for longest in (64, 3000):  # one slice, several
            lse = torch.full((sum(new), hq), float("nan"), device="cuda")
            out = p.cache.attend(dev(q, "bf16"), longest, cu_tokens=torch.from_numpy(cu).cuda(), max_new=max(new),
                                 window=window, sinks=sinks, lse=lse)
            torch.cuda.synchronize()
            check_attend(p, q, out, lse, cu, window, sinks, d ** -0.5, (rise, size, longest), max(new))


# ---------------------------------------------------------------- gains' gradients

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_gain_gradients_of_millions_of_tokens(gpu, dtype):
    """Four million equal tokens of 16 heads (the same row read with strides of
    0): every partial sum of a chain rounds the same way, so an error that grows
    with its length shows. Per element: a term 40 E; chains of 64 rows and those
    of one step, the sums of a workgroup in 64 bits, one rounding, then 768
    workgroups' sums in chains of 6, a tree of 3 and 16 streams: 40 + 66 + 1 + 25
    and some, 136 E of the terms' magnitudes."""
    import torch
    B = gpu
    rng = np.random.default_rng(22)
    t, hq, d = 1 << 22, 16, 64
    if dtype == "fp32":
        t //= 2
        hq *= 2
    cfg = B.heads_config(hq, 1, d, dtype=dtype, rot_dim=0)
    rows = {x: draw(rng, (1, 1, d), dtype) for x in ("q", "k", "dq", "dk")}
    gamma = draw(rng, d, dtype)
    wide = {x: dev(a, dtype).expand(t, 1 if "k" in x else hq, d) for x, a in rows.items()}
    got = B.qk_norm_rope_backward(cfg, {"gamma_q": dev(gamma, dtype), "gamma_k": dev(gamma, dtype)}, wide["q"], wide["k"],
                                  None, wide["dq"], wide["dk"])
    torch.cuda.synchronize()
    for i, (x, n) in enumerate((("q", t * hq), ("k", t))):
        dx, dg, mag, dg_mag = O.norm_rope_backward(rows[x], gamma, 1e-6, True, np.zeros((1, 0)), 0, False, rows["d" + x])
        first = got[i][:1, :1]
        close(host(first), dx, U[dtype] * np.abs(dx) + 64 * E * mag, (x, "dx"))
        assert torch.equal(got[i], first.expand_as(got[i]))
        close(host(got[2 + i]), n * dg, 136 * E * n * dg_mag, (x, "gain"))


# ---------------------------------------------------------------- angles

@pytest.mark.parametrize("pos", [1, 12345, -(1 << 20)])
def test_turns_near_the_axes(gpu, pos):
    """Angles next to whole quarter turns, whose sine or cosine is close to 0:
    the small one keeps its own digits. Rows (1, 0) of every pair give (cos,
    sin). Per element: 16 E of itself (cosine and sine 4 E, doubled where what
    fp32 leaves of the angle cancels half of it, and that term's roundings) and
    the angle's three roundings in 64 bits, 4 x 2^-53 of it."""
    import torch
    B = gpu
    d = 64
    cfg = B.heads_config(1, 1, d, dtype="fp32", norm=False)
    rng = np.random.default_rng(23)
    quarter = np.arange(d // 2) % 8 + abs(pos) - 1  # close to whole quarters, of every sign and distance
    ang = quarter * (np.pi / 2) + rng.standard_normal(d // 2) * 10.0 ** -(np.arange(d // 2) % 7 + 2)
    freqs = ang / pos
    x = torch.zeros(1, 1, d, device="cuda")
    x[..., :d // 2] = 1
    at = torch.full((1, 1), pos, dtype=torch.int32, device="cuda")
    got = B.qk_norm_rope_forward(cfg, {"freqs": torch.from_numpy(freqs).cuda()}, x, x, at)
    torch.cuda.synchronize()
    ang = pos * freqs
    ref = np.concatenate([np.cos(ang), np.sin(ang)])
    for y in got:
        close(host(y)[0, 0], ref, 16 * E * np.abs(ref) + 4 * 2.0 ** -53 * np.abs(np.concatenate([ang, ang])), pos)


# ---------------------------------------------------------------- what a cache holds

def test_cache_keeps_its_weights(gpu):
    """A cache goes on with the config, gains and frequencies that it was made
    with when the caller changes the config, or empties the dict or gives it
    others."""
    import gc
    import weakref
    import torch
    p = Paged(gpu, np.random.default_rng(24), 4, 2, 64, "bf16", 16, [20], [20], norm=True, rot=64)
    w = {name: t.clone() for name, t in p.weights.items()}
    cache = gpu.PagedCache(p.cfg, w, p.kd, p.vd, p.td, p.ld)
    held = {name: weakref.ref(t) for name, t in w.items()}
    w["gamma_q"] = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    del w["gamma_k"], w["freqs"]
    gc.collect()
    p.cfg.head_dim = 128
    assert cache.cfg.head_dim == 64
    assert all(r() is not None for r in held.values()), [n for n, r in held.items() if r() is None]


# ---------------------------------------------------------------- layouts

@pytest.mark.parametrize("t", [1, 33])
@pytest.mark.parametrize("order", ["head", "part"])
def test_projections_with_interleaved_heads(gpu, order, t):
    """q, k and v of one buffer whose heads hold their three rows side by side
    ([T, H, 3, D]), or whose rows hold their heads heads-first ([3, H, T, D]):
    normed and turned in place, forward, backward and append, as apart."""
    import torch
    B = gpu
    rng = np.random.default_rng(25)
    h, d, page = 6, 64, 16
    cfg = B.heads_config(h, h, d)
    w = {"gamma_q": dev(draw(rng, d, "bf16"), "bf16"), "gamma_k": dev(draw(rng, d, "bf16"), "bf16"),
         "freqs": B.rope_freqs(cfg)}
    pos = torch.arange(t, dtype=torch.int32, device="cuda")

    def buffer():
        if order == "head":
            b = dev(draw(rng, (t, h, 3, d), "bf16"), "bf16")
            return b, b.unbind(2)
        b = dev(draw(rng, (3, h, t, d), "bf16"), "bf16")
        return b, [x.transpose(0, 1) for x in b.unbind(0)]

    whole, (q, k, v) = buffer()
    grads, (dq, dk, _) = buffer()
    apart = [x.contiguous().clone() for x in (q, k, v, dq, dk)]
    want = B.qk_norm_rope_forward(cfg, w, apart[0], apart[1], pos)
    want_d = B.qk_norm_rope_backward(cfg, w, apart[0], apart[1], pos, apart[3], apart[4])
    got_d = B.qk_norm_rope_backward(cfg, w, q, k, pos, dq, dk, dq=dq, dk=dk)
    for x, y in zip(got_d, want_d):
        assert torch.equal(x, y)

    def cache():
        pages = [torch.zeros(4, h, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        return pages, B.PagedCache(cfg, w, *pages, torch.arange(4, dtype=torch.int32, device="cuda")[None],
                                   torch.tensor([t], dtype=torch.int32, device="cuda"))

    cu = torch.tensor([0, t], dtype=torch.int32, device="cuda")
    pages, c = cache()
    want_q = c.append(apart[1], apart[2], q=apart[0], cu_tokens=cu)
    pages2, c2 = cache()
    keep = whole.clone()
    got_q = c2.append(k, v, q=q, cu_tokens=cu, q_out=q)
    torch.cuda.synchronize()
    assert torch.equal(got_q, want_q) and all(torch.equal(x, y) for x, y in zip(pages, pages2))
    whole.copy_(keep)
    B.qk_norm_rope_forward(cfg, w, q, k, pos, q, k)
    torch.cuda.synchronize()
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, apart[2])


# ---------------------------------------------------------------- many tokens

def one_token_per_wave(t, d, *heads):
    """Whether a call takes a token per wave: 2,048 tokens or more whose rows fill
    the wave's passes of 1024 / head_dim rows to two thirds."""
    passes = sum(-(-h * d // 1024) for h in heads)
    return t >= 2048 and 2 * passes * (1024 // d) <= 3 * sum(heads)


MANY = {
    # as in test_gpu_heads.CASES; each fills its passes
    "T2048_h16_16x64": (2048, 16, 16, 64, "bf16", True, 64, False, (32,), "band"),
    "T2055_h16_4x128_pairs": (2055, 16, 4, 128, "bf16", True, 128, True, (20, 30, 14), "plain"),
    "T2051_h16x64_fp32_pairs": (2051, 16, 16, 64, "fp32", True, 48, True, (24,), "heads"),
    "T2049_h16_8x128_fp32": (2049, 16, 8, 128, "fp32", True, 128, False, (64,), "band"),
    "T2050_h32_16x64_no_norm": (2050, 32, 16, 64, "bf16", False, 32, True, (16,), "plain"),
}


@pytest.mark.parametrize("name", MANY)
def test_forward_of_many_tokens(gpu, name):
    import torch
    t, hq, hk, d, dtype, norm, rot, pairs, axes, layout = MANY[name]
    assert one_token_per_wave(t, d, hq, hk)
    a = qk_inputs(gpu, MANY[name], 26)
    got = gpu.qk_norm_rope_forward(a["cfg"], a["w"], laid_out(a["q"], dtype, layout), laid_out(a["k"], dtype, layout), a["pos"])
    torch.cuda.synchronize()
    for y, x, g in ((got[0], a["q"], a["g"][0]), (got[1], a["k"], a["g"][1])):
        ref, mag = O.norm_rope(x, g, 1e-5, norm, a["ang"], rot, pairs)
        close(host(y), ref, U[dtype] * np.abs(ref) + 32 * E * mag, name)


STEPS = {
    # 768 workgroups of eight tokens: 6,144 in a step of the backward
    "T6144_h4_2x64": (6144, 4, 2, 64, "bf16", True, 64, False, (32,), "plain"),
    "T6151_h5_1x128_fp32_pairs": (6151, 5, 1, 128, "fp32", True, 128, True, (64,), "band"),
    "T13001_h4_4x64_axes": (13001, 4, 4, 64, "bf16", True, 32, False, (5, 11), "heads"),
    "T12289_h3x64_fp32_no_norm": (12289, 3, 3, 64, "fp32", False, 64, False, (32,), "plain"),
    "T6145_h20x128": (6145, 20, 20, 128, "bf16", True, 128, False, (64,), "plain"),
}


@pytest.mark.parametrize("name", STEPS)
def test_backward_of_several_steps(gpu, name):
    import torch
    t, hq, hk, d, dtype, norm, rot, pairs, axes, layout = STEPS[name]
    a = qk_inputs(gpu, STEPS[name], 27)
    x = {n: laid_out(a[n], dtype, layout) for n in ("q", "k", "dq", "dk")}
    got = gpu.qk_norm_rope_backward(a["cfg"], a["w"], x["q"], x["k"], a["pos"], x["dq"], x["dk"])
    again = gpu.qk_norm_rope_backward(a["cfg"], a["w"], x["q"], x["k"], a["pos"], x["dq"], x["dk"], dq=x["dq"], dk=x["dk"])
    torch.cuda.synchronize()
    for y, z in zip(got, again):
        assert (y is None and z is None) or torch.equal(y, z)
    for i, n in enumerate(("q", "k")):
        dx, dg, mag, dg_mag = O.norm_rope_backward(a[n], a["g"][i], 1e-5, norm, a["ang"], rot, pairs, a["d" + n])
        close(host(got[i]), dx, U[dtype] * np.abs(dx) + 64 * E * mag, (name, n))
        if norm:
            close(host(got[2 + i]), dg, 128 * E * dg_mag, (name, "gain", n))


@pytest.mark.parametrize("case", [(32, 8, 128, "bf16", 16, False), (16, 16, 64, "fp32", 48, True), (16, 4, 128, "bf16", 64, True)],
                         ids=str)
def test_append_of_many_tokens(gpu, case):
    """Prompts of more than 2,048 tokens together, with padding behind them, a
    token per wave: rows of the pages and queries against the oracle, the rest
    as it was."""
    import torch
    hq, hk, d, dtype, page, pairs = case
    rng = np.random.default_rng(28)
    lens, new, pad = [1500, 40, 900, 16], [1400, 0, 700, 16], 9
    p = Paged(gpu, rng, hq, hk, d, dtype, page, lens, [0] * 4, norm=True, rot=d, pairs=pairs)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    t = int(cu[-1]) + pad
    assert one_token_per_wave(t, d, hq, hk, hk)
    q, k, v = draw(rng, (t, hq, d), dtype), draw(rng, (t, hk, d), dtype), draw(rng, (t, hk, d), dtype)
    qo = torch.full((t, hq, d), 7.0, dtype=p.kd.dtype, device="cuda")
    cud = torch.from_numpy(cu).cuda()
    p.cache.append(laid_out(k, dtype, "band"), laid_out(v, dtype, "heads"), q=laid_out(q, dtype, "band"), q_out=qo, cu_tokens=cud)
    kd, vd = p.kd.clone(), p.vd.clone()
    p.kd.fill_(float("nan")), p.vd.fill_(float("nan"))
    p.cache.append(dev(k, dtype), dev(v, dtype), cu_tokens=cud)  # without queries: 4 + 4 heads take four tokens
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(p.kd.view(bits), kd.view(bits)) and torch.equal(p.vd.view(bits), vd.view(bits))
    rows = O.token_rows(lens, cu)
    n = len(rows)
    ang = O.angles([[r for _, r in rows]], p.weights["freqs"].cpu().numpy(), [d // 2])
    at = np.array([O.place(p.table[s], r, page, p.n_pages) for s, r in rows])
    got_q, got_k, got_v = host(qo), host(kd), host(vd)
    for x, g, y in ((q, p.gammas[0], got_q[:n]), (k, p.gammas[1], got_k[at[:, 0], :, at[:, 1]])):
        ref, mag = O.norm_rope(x[:n], g, 1e-6, True, ang, d, pairs)
        close(y, ref, U[dtype] * np.abs(ref) + 32 * E * mag, case)
    assert (got_q[n:] == 7).all() and np.array_equal(got_v[at[:, 0], :, at[:, 1]], v[:n])
    untouched = np.ones((p.n_pages, page), bool)
    untouched[at[:, 0], at[:, 1]] = False
    assert np.isnan(got_k.transpose(0, 2, 1, 3)[untouched]).all() and np.isnan(got_v.transpose(0, 2, 1, 3)[untouched]).all()
