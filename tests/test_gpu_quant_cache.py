"""The 8-bit cache on the GPU against the float64 oracle: append, read back and
attention over it, alone and as they are used together.

Rows that are not normed or turned are held and read back without any
tolerance: scales are powers of two and each element is rounded once. Normed or
turned keys come within half a step of their own norm and rotation: 2^-4 of the
value or half the smallest step, 2^-10 of the row's power of two (which is at
most the top magnitude over 224, or twice that where rounding takes the top
over a border: 2^-9 / 224), after the norm's own 32 E m. Attention has the
tolerances of the paged cache's (test_gpu_heads.py) over the values that the
rows stand for.
"""
import numpy as np
import pytest

from oracle import heads as O
from helpers import dev, host
from test_gpu_heads import E, U, close, draw, laid_out

pytestmark = pytest.mark.gpu


def pool(n_pages, hk, page, d):
    """Pages and scales that hold NaN codes and scale bytes of 255."""
    import torch
    codes = [torch.full((n_pages, hk, page, d), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "kv"]
    return codes + [torch.full((n_pages, hk, page), 255, dtype=torch.uint8, device="cuda") for _ in "kv"]


def values(codes, scales):
    x = codes.float().cpu().double().numpy()
    return x * np.exp2(scales.cpu().double().numpy() - 127)[..., None]


def set_up(B, lens, news, hq, hk, d, dtype, page, norm=False, rot=0, style=0, seed=1, spare=3, lost=()):
    """A cache of sequences of `lens` rows whose last `news` are new, and the
    new tokens' rows; `lost`: (sequence, page) entries that are no page."""
    import torch
    rng = np.random.default_rng(seed)
    cfg = B.heads_config(hq, hk, d, dtype=dtype, norm=norm, eps=1e-5, rot_dim=rot, style=style)
    pages = [-(-max(n, 0) // page) for n in lens]
    n_pages = sum(pages) + spare
    order = rng.permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), max(pages) + 1), -1, np.int32)
    at = 0
    for s, p in enumerate(pages):
        table[s, :p] = order[at:at + p]
        at += p
    for i, (s, p) in enumerate(lost):
        table[s, p] = (-5, n_pages, 2**31 - 1)[i % 3]
    w = {"gamma_q": None, "gamma_k": None, "freqs": B.rope_freqs(cfg) if rot else None}
    g = [None, None]
    if norm:
        g = [draw(rng, d, dtype) * 0.25 + 1 for _ in range(2)]
        g = [host(dev(x, dtype)) for x in g]
        w["gamma_q"], w["gamma_k"] = (dev(x, dtype) for x in g)
    p = pool(n_pages, hk, page, d)
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cache = B.PagedCache8(cfg, w, *p, torch.from_numpy(table).cuda(), kv_len)
    cu = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    t = int(cu[-1])
    rows = {n: draw(rng, (t, h, d), dtype, s) for n, h, s in (("q", hq, 2), ("k", hk, 1), ("v", hk, 3))}
    for n in "kv":  # rows of very different magnitudes
        rows[n] *= np.exp2(rng.integers(-20, 20, rows[n].shape[:2]))[..., None].astype(np.float32)
    return dict(cfg=cfg, cache=cache, pool=p, table=table, lens=lens, news=news, cu=cu, t=t, rows=rows, g=g, w=w,
                n_pages=n_pages, page=page, dtype=dtype, kv_len=kv_len, cu_gpu=torch.from_numpy(cu).cuda())


CASES = {
    # name: (rows, new ones, heads, kv heads, head_dim, dtype, page, norm, rot, style, layout, lost pages)
    "one_token": ([1], [1], 2, 1, 64, "bf16", 16, False, 0, 0, "plain", ()),
    "tokens": ([40, 1, 17, 33], [1, 1, 1, 1], 8, 2, 128, "bf16", 32, False, 0, 0, "band", ()),
    "tokens_fp32": ([40, 1, 17, 33], [1, 1, 1, 1], 3, 3, 64, "fp32", 16, False, 0, 0, "heads", ()),
    "prompts": ([70, 30, 0, 129], [70, 5, 0, 100], 4, 4, 64, "bf16", 48, False, 0, 0, "plain", ()),
    "prompts_fp32": ([70, 30, 129], [69, 30, 1], 5, 5, 128, "fp32", 16, False, 0, 0, "band", ()),
    "lost_pages": ([70, 90, 40], [70, 90, 40], 2, 2, 64, "bf16", 16, False, 0, 0, "plain", ((0, 1), (1, 0), (1, 5))),
    "before_row_0": ([10, 3], [15, 4], 2, 1, 128, "bf16", 16, False, 0, 0, "plain", ()),
    "normed": ([70, 30, 129], [70, 30, 128], 6, 3, 128, "bf16", 32, True, 128, 0, "band", ()),
    "normed_pairs_fp32": ([33, 64], [30, 64], 4, 1, 64, "fp32", 16, True, 32, 1, "plain", ()),
    "turned_only": ([50], [50], 4, 4, 64, "bf16", 16, False, 64, 0, "heads", ()),
    "many_tokens": ([3000, 700], [2900, 700], 4, 2, 64, "bf16", 64, True, 64, 0, "plain", ()),
}


@pytest.mark.parametrize("name", CASES)
def test_append_and_read(gpu, name):
    import torch
    lens, news, hq, hk, d, dtype, page, norm, rot, style, layout, lost = CASES[name]
    a = set_up(gpu, lens, news, hq, hk, d, dtype, page, norm, rot, style, lost=lost)
    q, k, v = (laid_out(a["rows"][n], dtype, layout) for n in "qkv")
    cu = None if name.startswith("tokens") else a["cu_gpu"]
    q_out = torch.full(q.shape, 5.0, dtype=q.dtype, device="cuda")
    a["cache"].append(k, v, q=q, cu_tokens=cu, q_out=q_out)
    back = [torch.full((a["t"], hk, d), 5.0, dtype=q.dtype, device="cuda") for _ in "kv"]
    assert a["cache"].read(*back, cu_tokens=cu) == tuple(back)
    torch.cuda.synchronize()
    freqs = a["w"]["freqs"].cpu().numpy() if rot else np.zeros(0)
    held = [values(a["pool"][i], a["pool"][2 + i]) for i in range(2)]
    touched = np.zeros((a["n_pages"], page), bool)
    for t, (s, row) in enumerate(O.token_rows(lens, a["cu"])):
        pl = O.place(a["table"][s], row, page, a["n_pages"])
        if pl is None:
            assert (host(q_out)[t] == 5).all() and all((host(b)[t] == 5).all() for b in back)
            continue
        touched[pl] = True
        ang = O.angles([[row]], freqs, (rot // 2,)) if rot else np.zeros((1, 0))
        for i, n in enumerate("kv"):
            got, byte = held[i][pl[0], :, pl[1]], a["pool"][2 + i][pl[0], :, pl[1]].cpu().numpy()
            np.testing.assert_array_equal(host(back[i])[t], got, err_msg=str((name, t, n)))
            x = a["rows"][n][t:t + 1]
            if n == "v" or (not norm and not rot):
                want, want_byte = O.quantised(x.astype(np.float64))
                np.testing.assert_array_equal(got, want[0], err_msg=str((name, t, n)))
                np.testing.assert_array_equal(byte, want_byte[0])
            else:
                ref, mag = O.norm_rope(x, a["g"][1], 1e-5, norm, ang, rot, bool(style))
                top = np.abs(ref[0]).max(-1, keepdims=True)
                tol = 2.0 ** -4 * np.abs(ref[0]) + 2.0 ** -9 / 224 * top + (1 + 2.0 ** -4) * 32 * E * mag[0]
                close(got, ref[0], tol, (name, t))
        ref, mag = O.norm_rope(a["rows"]["q"][t:t + 1], a["g"][0], 1e-5, norm, ang, rot, bool(style))
        close(host(q_out)[t], ref[0], U[dtype] * np.abs(ref[0]) + 32 * E * mag[0], (name, t, "q"))
    for i in range(2):  # all other rows as they were
        rest = np.broadcast_to(~touched[:, None], (a["n_pages"], hk, page))
        assert np.isnan(held[i][rest]).all()
        assert (a["pool"][2 + i].cpu().numpy()[rest] == 255).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [64, 128])
def test_edges_of_the_format(gpu, dtype, d):
    """Every code and every tie between codes, tops at both sides of a power of
    two, zeros, the type's smallest and largest values, infinities and NaN."""
    import torch
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    pos = np.unique(np.abs(codes[np.isfinite(codes)]))
    ties = (pos[1:] + pos[:-1]) / 2
    big = 3.3895313892515355e38 if dtype == "bf16" else 3.4028234663852886e38
    rows = []
    for x in (pos, -pos, ties, -ties):
        for part in np.array_split(x, 4):
            rows.append(np.concatenate([part, np.full(d - len(part) - 1, 0.0), [448.0]]))
    for top in (448.0, 450.0, 224.0, 225.0, 1.0, 1.75, 1.7578125, 2.0 ** -100, 2.0 ** -126, 2.0 ** -133, 1.5 * 2.0 ** 100, 2.0 ** 127):
        rows.append(np.concatenate([[top], top * np.linspace(-1, 1, d - 1)]))
    rows += [np.zeros(d), np.full(d, -0.0), np.full(d, np.inf), np.full(d, np.nan),
             np.concatenate([[np.inf, -np.inf, np.nan, 3.0], np.linspace(-1, 1, d - 4)]), np.full(d, big), np.full(d, -big / 2)]
    x = np.stack(rows).astype(np.float32)[:, None]
    x = host(dev(x, dtype))
    t = len(x)
    a = set_up(gpu, [t], [t], 1, 1, d, dtype, 16)
    k, v = dev(x.astype(np.float32), dtype), dev(x[::-1].astype(np.float32), dtype)
    a["cache"].append(k, v, cu_tokens=a["cu_gpu"])
    back = [torch.empty((t, 1, d), dtype=k.dtype, device="cuda") for _ in "kv"]
    a["cache"].read(*back, cu_tokens=a["cu_gpu"])
    for got, y in zip(back, (x, x[::-1])):
        want, byte = O.quantised(y)
        assert byte.min() == 17 and byte.max() == 247
        with np.errstate(over="ignore"):  # 256 * 2^120 is past both types
            want = want.astype(np.float32).astype(np.float64)
        np.testing.assert_array_equal(host(got), want)


ATTEND = {
    # name: (rows, new ones, heads, kv heads, head_dim, dtype, page, window, sinks, max_new, lost pages)
    "one_row": ([1, 2], [1, 1], 2, 1, 64, "bf16", 16, 0, 0, 1, ()),
    "tile_edges": ([15, 16, 17, 63, 64, 65, 127, 129, 257], [1] * 9, 4, 2, 128, "bf16", 16, 0, 0, 1, ()),
    "tile_edges_fp32": ([15, 16, 17, 63, 64, 65, 129], [1] * 7, 4, 2, 64, "fp32", 48, 0, 0, 1, ()),
    "empty_slots": ([0, 40, -3, 500], [1] * 4, 2, 2, 64, "bf16", 32, 0, 0, 1, ()),
    "group_of_40": ([300], [1], 40, 1, 128, "bf16", 16, 0, 0, 1, ()),
    "slices": ([5000, 1, 2500], [1] * 3, 4, 1, 64, "bf16", 64, 0, 0, 1, ()),
    "slices_fp32": ([3000, 700], [1] * 2, 4, 2, 128, "fp32", 64, 0, 0, 1, ()),
    "window": ([900, 30, 200], [1] * 3, 4, 2, 64, "bf16", 16, 100, 5, 1, ()),
    "window_1_fp32": ([90, 3], [1] * 2, 2, 2, 128, "fp32", 16, 1, 0, 1, ()),
    "few_tokens": ([70, 30, 129], [7, 30, 20], 4, 2, 128, "bf16", 16, 0, 0, 31, ()),
    "prompts": ([170, 30, 0, 329], [100, 30, 0, 65], 4, 2, 64, "bf16", 48, 0, 0, 100, ()),
    "prompts_128": ([170, 64, 640], [130, 64, 65], 8, 2, 128, "bf16", 16, 0, 0, 130, ()),
    "prompts_window": ([500, 900], [300, 40], 4, 4, 64, "bf16", 32, 70, 33, 300, ()),
    "prompts_window_128": ([500, 900], [300, 40], 5, 1, 128, "bf16", 16, 70, 3, 300, ()),
    "prompts_fp32": ([100, 90], [50, 90], 4, 2, 64, "fp32", 16, 20, 2, 90, ()),
    "long_prompt_pages": ([2200], [40], 2, 1, 64, "bf16", 16, 0, 0, 40, ()),
    "lost_pages": ([300, 200], [1, 1], 2, 2, 64, "bf16", 16, 0, 0, 1, ((0, 0), (0, 7), (1, 12))),
    "lost_pages_prompt": ([300, 200], [64, 200], 2, 2, 128, "bf16", 16, 0, 0, 200, ((0, 0), (0, 7), (1, 12))),
}


@pytest.mark.parametrize("name", ATTEND)
def test_attention(gpu, name):
    """Rows that no token sees hold NaN codes and scale bytes of 255."""
    import torch
    lens, news, hq, hk, d, dtype, page, window, sinks, max_new, lost = ATTEND[name]
    a = set_up(gpu, lens, news, hq, hk, d, dtype, page, lost=lost, seed=2)
    rng = np.random.default_rng(3)
    whole = [max(n, 0) for n in lens]
    cu_all = torch.tensor(np.concatenate([[0], np.cumsum(whole)]).astype(np.int32), device="cuda")
    k, v = (dev(draw(rng, (sum(whole), hk, d), dtype), dtype) for _ in range(2))
    a["cache"].append(k, v, cu_tokens=cu_all)
    if window:  # what windows never reach
        for s, (n, new) in enumerate(zip(lens, news)):
            for row in range(sinks, n - new - window + 1):
                pl = O.place(a["table"][s], row, page, a["n_pages"])
                for i in range(2):
                    a["pool"][i].view(torch.uint8)[pl[0], :, pl[1]] = 0x7F
                    a["pool"][2 + i][pl[0], :, pl[1]] = 255
    q = dev(a["rows"]["q"], dtype)
    cu = None if max_new == 1 else a["cu_gpu"]
    lse = torch.full((a["t"], hq), 5.0, device="cuda")
    out = a["cache"].attend(q, max(max(lens), 1), cu_tokens=cu, max_new=max_new, window=window, sinks=sinks, lse=lse)
    torch.cuda.synchronize()
    held = [values(a["pool"][i], a["pool"][2 + i]) for i in range(2)]
    ref, rl, err, mag = O.paged_attention(a["rows"]["q"], *held, a["table"], lens, a["cu"], d ** -0.5, window, sinks)
    n = max(max(lens), 1)
    score = (d + 10) * E * err + 8 * E
    r = 0.0 if dtype == "fp32" else 2.0 ** -8 if max_new >= 32 else 2.0 ** -17
    close(host(out), ref, U[dtype] * np.abs(ref) + (2 * score + (n + 64) * E + r)[..., None] * mag, name)
    sees = np.isfinite(rl)
    close(host(lse)[sees], rl[sees], (2 * score + (n + 64) * E + 4 * E * np.abs(rl))[sees], (name, "lse"))
    assert (host(lse)[~sees] == -np.inf).all()
    again = a["cache"].attend(q, max(max(lens), 1), cu_tokens=cu, max_new=max_new, window=window, sinks=sinks)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_conversation(gpu, dtype):
    """A prompt taken whole by the packed attention while its keys and values
    go into the 8-bit cache, then token after token over it, eager and as a
    captured step; what the cache holds read back whole and attended again by
    the packed attention: both see the same values, so the last token's results
    differ by both sides' tolerances alone."""
    import torch
    hq, hk, d, page, n0, steps = 4, 2, 64, 16, 75, 6
    cfg = gpu.heads_config(hq, hk, d, dtype=dtype, eps=1e-5)
    rng = np.random.default_rng(11)
    w = {"gamma_q": dev(draw(rng, d, dtype, 0.1) + 1, dtype), "gamma_k": dev(draw(rng, d, dtype, 0.1) + 1, dtype),
         "freqs": gpu.rope_freqs(cfg)}
    p = pool(20, hk, page, d)
    table = torch.from_numpy(rng.permutation(20)[:2 * 8].reshape(2, 8).astype(np.int32)).cuda()
    kv_len = torch.tensor([n0, n0 - 20], dtype=torch.int32, device="cuda")
    cache = gpu.PagedCache8(cfg, w, *p, table, kv_len)
    lens = [n0, n0 - 20]
    cu = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device="cuda")
    qkv = dev(draw(rng, (sum(lens), hq + 2 * hk, d), dtype), dtype)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    pos = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
    qt, kt = gpu.qk_norm_rope_forward(cfg, w, q, k, pos)
    whole, _ = gpu.packed_attention_forward(cfg, qt, kt, v, cu, n0)
    qa = cache.append(k, v, q=q, cu_tokens=cu)
    assert torch.equal(qa, qt) and torch.isfinite(whole).all()
    tok = torch.empty(2, hq + 2 * hk, d, dtype=qkv.dtype, device="cuda")
    q_out, out = torch.empty(2, hq, d, dtype=qkv.dtype, device="cuda"), torch.empty(2, hq, d, dtype=qkv.dtype, device="cuda")

    def step():
        cache.append(tok[:, hq:hq + hk], tok[:, hq + hk:], q=tok[:, :hq], q_out=q_out)
        cache.attend(q_out, n0 + steps, out=out)

    step()  # (overwrites the last rows with rows of its own: appended again below)
    cache.append(k, v, q=q, cu_tokens=cu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(steps):
        kv_len += 1
        tok.copy_(dev(draw(rng, tuple(tok.shape), dtype), dtype))
        graph.replay()
        torch.cuda.synchronize()
        seen = out.clone()
        step()
        assert torch.equal(seen, out)
        lens = [n + 1 for n in lens]
    ends = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device="cuda")
    kr, vr = (torch.empty(sum(lens), hk, d, dtype=qkv.dtype, device="cuda") for _ in range(2))
    cache.read(kr, vr, cu_tokens=ends)
    qs = torch.zeros(sum(lens), hq, d, dtype=qkv.dtype, device="cuda")
    last = [lens[0] - 1, sum(lens) - 1]
    qs[last] = q_out
    packed, _ = gpu.packed_attention_forward(cfg, qs, kr, vr, ends, max(lens))
    ref, _, err, mag = O.packed_attention(host(qs), host(kr), host(vr), ends.cpu().numpy(), d ** -0.5)
    n = max(lens)
    for got, w_ in ((packed[last], 2.0 ** -8), (out, 2.0 ** -17)):
        tol = U[dtype] * np.abs(ref[last]) + (2 * ((d + 10) * E * err + 8 * E) + (n + 64) * E + (w_ if dtype == "bf16" else 0))[last][..., None] * mag[last]
        close(host(got), ref[last], tol, dtype)


def test_far_pages(gpu):
    """A pool of more than 4 GiB per tensor: offsets past 32 bits."""
    import torch
    hk, page, d = 1, 16, 128
    n_pages = (5 << 30) // (hk * page * d)
    cfg = gpu.heads_config(2, hk, d, norm=False, rot_dim=0)
    codes = [torch.empty((n_pages, hk, page, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "kv"]
    scales = [torch.empty((n_pages, hk, page), dtype=torch.uint8, device="cuda") for _ in "kv"]
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, n_pages // 2, n_pages - 7, 1]], dtype=torch.int32, device="cuda")
    kv_len = torch.tensor([90], dtype=torch.int32, device="cuda")
    cache = gpu.PagedCache8(cfg, {}, *codes, *scales, table, kv_len)
    rng = np.random.default_rng(12)
    x = {n: draw(rng, (90, h, d), "bf16") for n, h in (("q", 2), ("k", 1), ("v", 1))}
    cu = torch.tensor([0, 90], dtype=torch.int32, device="cuda")
    cache.append(dev(x["k"], "bf16"), dev(x["v"], "bf16"), cu_tokens=cu)
    kr, vr = (torch.empty(90, 1, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.read(kr, vr, cu_tokens=cu)
    np.testing.assert_array_equal(host(kr), O.quantised(x["k"])[0])
    np.testing.assert_array_equal(host(vr), O.quantised(x["v"])[0])
    one = cache.attend(dev(x["q"], "bf16")[-1:], 90)
    all_ = cache.attend(dev(x["q"], "bf16"), 90, cu_tokens=cu)
    ref, _, err, mag = O.packed_attention(x["q"], host(kr), host(vr), [0, 90], d ** -0.5)
    tol = lambda r: U["bf16"] * np.abs(ref) + (2 * ((d + 10) * E * err + 8 * E) + 154 * E + r)[..., None] * mag  # noqa: E731
    close(host(all_), ref, tol(2.0 ** -8), "prompt")
    close(host(one), ref[-1:], tol(2.0 ** -17)[-1:], "token")


def test_the_binding_refuses(gpu):
    import torch
    cfg = gpu.heads_config(4, 2, 64)
    w = {"freqs": gpu.rope_freqs(cfg)}
    good = dict(zip(("k_pages", "v_pages", "k_scales", "v_scales"), pool(4, 2, 16, 64)), page_table=torch.zeros(1, 4, dtype=torch.int32, device="cuda"),
                kv_len=torch.zeros(1, dtype=torch.int32, device="cuda"))
    gpu.PagedCache8(cfg, w, **good)
    for bad in (dict(k_pages=good["k_pages"].view(torch.uint8)), dict(v_pages=good["v_pages"].float()), dict(k_scales=good["k_scales"][:3]),
                dict(v_scales=good["v_scales"].float()), dict(k_scales=good["k_scales"].cpu()), dict(v_scales=good["v_scales"].transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            gpu.PagedCache8(cfg, w, **dict(good, **bad))
    cache = gpu.PagedCache8(cfg, w, **good)
    r = lambda h, dt=torch.bfloat16: torch.zeros(1, h, 64, dtype=dt, device="cuda")  # noqa: E731
    for k, v in ((r(4), r(2)), (r(2, torch.float32), r(2)), (r(2), r(2).cpu())):
        with pytest.raises(ValueError):
            cache.read(k, v)
    with pytest.raises(ValueError):
        gpu.PagedCache(cfg, w, good["k_pages"], good["v_pages"], good["page_table"], good["kv_len"])
