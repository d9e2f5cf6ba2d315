"""The launch orders that large calls take: blocks of columns dealt by weight over
sequences (2 to 64 of them, 512 workgroups and more), K/V heads in multiples of
the XCDs and not, several rounds of workgroups with a part of one left over, the
cuts of the backward's queries, and reads and appends of many tokens. Every output
is compared with the definition in float64 on the GPU, within the tolerances of
test_gpu_packed.py and test_gpu_heads.py.
"""
import numpy as np
import pytest

from helpers import torch_dtype
from test_gpu_heads import E, U

pytestmark = pytest.mark.gpu


def attention64(q, k, v, row0, scale, window=0, sinks=0):
    """(weights, out, lse, score error scale, value magnitude) of one head's tokens
    q [n, D] at rows row0 .. of k, v [rows, D], as in oracle.heads."""
    import torch
    row, j = row0 + torch.arange(len(q), device="cuda")[:, None], torch.arange(len(k), device="cuda")[None]
    seen = j <= row
    if window:
        seen &= (j > row - window) | (j < sinks)
    s = (scale * (q @ k.T)).masked_fill(~seen, -np.inf)
    top = s.amax(-1, keepdim=True)
    p = (s - top).exp()
    total = p.sum(-1, keepdim=True)
    p /= total
    err = (abs(scale) * (q.abs() @ k.abs().T)).masked_fill(~seen, 0).amax(-1)
    return p, p @ v, (top + total.log())[:, 0], err, p @ v.abs()


def within(got, ref, tol, what):
    bad = ~((got.double() - ref).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], ref[bad][:4], tol[bad][:4])


PACKED = {
    # name: (lengths, heads, kv heads, head_dim, dtype, window, sinks, tokens behind, least and most column and key groups)
    "ranked_8": ([700, 0, 300, 1, 1100, 257], 32, 8, 64, "bf16", 0, 0, 40, (512, 1 << 20), (64, 511)),
    "ranked_8_fp32": ([700, 0, 300, 1, 1100, 257], 32, 8, 64, "fp32", 0, 0, 40, (512, 1 << 20), (64, 511)),
    "ranked_8x128_fp32": ([1201, 0, 900, 333], 32, 8, 128, "fp32", 0, 0, 3, (512, 1 << 20), (64, 511)),
    "ranked_16": ([1700, 1, 0, 900, 1100], 16, 16, 128, "bf16", 0, 0, 9, (512, 1 << 20), (512, 767)),
    "ranked_3": ([1500, 0, 1300, 1400, 1201], 12, 3, 64, "bf16", 0, 0, 0, (512, 1 << 20), (64, 511)),
    "ranked_group_of_5": ([900, 0, 700, 1000], 40, 8, 64, "bf16", 0, 0, 7, (512, 1 << 20), (64, 511)),
    "64_sequences": ([(i * 37) % 61 for i in range(64)], 16, 8, 64, "bf16", 0, 0, 11, (512, 1 << 20), (512, 767)),
    "65_sequences": ([(i * 37) % 61 for i in range(65)], 16, 8, 64, "bf16", 0, 0, 0, (512, 1 << 20), (512, 767)),
    "one_long_8": ([3000], 8, 8, 64, "bf16", 0, 0, 5, (1, 511), (64, 511)),
    "one_long_32_8": ([2500], 32, 8, 128, "bf16", 0, 0, 0, (512, 1 << 20), (64, 511)),
    "windowed_8": ([1300, 40, 900], 32, 8, 128, "bf16", 300, 5, 0, (512, 1 << 20), (64, 511)),
    "windowed_16_fp32": ([700, 0, 640], 16, 16, 64, "fp32", 150, 3, 20, (1, 511), (64, 511)),
    "two_slices": ([4100, 0, 2100, 2300], 32, 8, 64, "bf16", 0, 0, 0, (512, 1 << 20), (512, 767)),
    "two_slices_fp32": ([4100, 0, 2100, 2300], 32, 8, 64, "fp32", 0, 0, 0, (512, 1 << 20), (512, 767)),
    "long_lists": ([4100, 2100, 2300, 0, 2600, 1500], 32, 8, 64, "bf16", 0, 0, 13, (512, 1 << 20), (768, 1 << 20)),
    "long_lists_128": ([4100, 2100, 2300, 0, 2600, 1500], 16, 8, 128, "bf16", 0, 0, 0, (512, 1 << 20), (768, 1 << 20)),
    "windowed_lists": ([4100, 2100, 2300, 0, 2600, 1500], 16, 16, 64, "bf16", 600, 4, 0, (512, 1 << 20), (768, 1 << 20)),
}


@pytest.mark.parametrize("name", PACKED)
def test_packed(gpu, name):
    import torch
    lens, hq, hk, d, dtype, window, sinks, behind, columns, keys = PACKED[name]
    t, total = sum(lens), sum(lens) + behind
    blocks = total * (hq // hk) // 128 + len(lens)
    assert columns[0] <= blocks * hk <= columns[1] and keys[0] <= (total // 128 + len(lens)) * hk <= keys[1]
    torch.manual_seed(1)
    dt = torch_dtype(dtype)
    q, do = (torch.randn(total, hq, d, device="cuda").to(dt) for _ in range(2))
    k, v = (torch.randn(total, hk, d, device="cuda").to(dt) for _ in range(2))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    cfg = gpu.heads_config(hq, hk, d, dtype=dtype, norm=False, rot_dim=0)
    kw = dict(window=window, sinks=sinks)
    out, lse = gpu.packed_attention_forward(cfg, q, k, v, cu, max(lens), **kw)
    got = gpu.packed_attention_backward(cfg, q, k, v, out, lse, do, cu, max(lens), **kw)
    torch.cuda.synchronize()
    for y in (out, lse, *got):  # poisoned before the call
        assert torch.isnan(y[t:]).all() and torch.isfinite(y[:t]).all()
    n, u, scale, group = max(lens), U[dtype], d ** -0.5, hq // hk
    w = 2.0 ** -8 if dtype == "bf16" else 0.0
    sums = (n * group + 64) * E
    pe = (d + 10) * E + sums
    for a, b in zip(cu[:-1].tolist(), cu[1:].tolist()):
        for kv in range(hk if b > a else 0):
            ki, vi = k[a:b, kv].double(), v[a:b, kv].double()
            dk, dv, dk_tol, dv_tol = (torch.zeros_like(ki) for _ in range(4))
            for h in range(kv * group, (kv + 1) * group):
                qi, oi = q[a:b, h].double(), do[a:b, h].double()
                p, o, l, err, mag = attention64(qi, ki, vi, 0, scale, window, sinks)
                s = (d + 10) * E * err + 8 * E
                of_lse = 2 * s + (n + 64) * E + 4 * E * l.abs()
                of_out = u * o.abs() + (2 * s + (n + 64) * E + w)[:, None] * mag
                within(out[a:b, h], o, of_out, (name, "out", a, h))
                within(lse[a:b, h], l, of_lse, (name, "lse", a, h))
                # the gradients and their bounds, as oracle.heads.packed_attention_backward has them
                wt = (s + of_lse + 8 * E + 2 * E * (l.abs() + err) + sums)[:, None]
                dp = oi @ vi.T
                slope = dp - (p * dp).sum(-1, keepdim=True)
                ds = p * slope
                off = (oi.abs() * (of_out + pe * o.abs())).sum(-1, keepdim=True)
                e = p * (wt * slope.abs() + pe * (oi.abs() @ vi.abs().T) + off) * (1 + wt) * (1 + w) + (w + pe) * ds.abs()
                dq = scale * (ds @ ki)
                within(got[0][a:b, h], dq, u * dq.abs() + (1 + u) * scale * (e @ ki.abs()) + 2.0 ** -100, (name, "dq", a, h))
                dk += scale * (ds.T @ qi)
                dv += p.T @ oi
                dk_tol += scale * (e.T @ qi.abs())
                dv_tol += ((wt + w + wt * w + pe) * p).T @ oi.abs()
            within(got[1][a:b, kv], dk, u * dk.abs() + (1 + u) * dk_tol + 2.0 ** -100, (name, "dk", a, kv))
            within(got[2][a:b, kv], dv, u * dv.abs() + (1 + u) * dv_tol + 2.0 ** -100, (name, "dv", a, kv))


PROMPTS = {
    # name: (new tokens, rows behind which they come, heads, kv heads, head_dim, page, window, sinks, least workgroups, slices)
    "whole_8": ([700, 0, 300, 1, 900], [0, 50, 3000, 900, 100], 32, 8, 128, 32, 0, 0, 512, 1),
    "sliced_16": ([500, 200, 33, 300, 0], [100, 2000, 0, 900, 60], 16, 16, 64, 64, 0, 0, 512, 3),
    "sliced_3": ([500, 0, 400, 100, 300], [0, 2000, 1100, 5, 900], 12, 3, 64, 16, 0, 0, 512, 4),
    "one_8": ([1500], [2500], 8, 8, 128, 16, 0, 0, 1, 6),
    "windowed_8": ([600, 77, 0, 900], [1000, 30, 70, 0], 32, 8, 64, 48, 200, 5, 512, 2),
    "group_of_5": ([900, 0, 555], [70, 20, 700], 40, 8, 64, 16, 0, 0, 1, 2),
}


def filled(rows, hk, d, page, bits8, seed):
    """Pages whose slots are poisoned but for the sequences' rows, a table, and those
    rows' values [rows, hk, d] in 64 bits, of K and V."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pages = [-(-n // page) for n in rows]
    n_pages = sum(pages) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(rows), max(pages) + 1), -1, dtype=torch.int32, device="cuda")
    pool, held, first = [], [], 0
    for s, p in enumerate(pages):
        table[s, :p] = order[first:first + p]
        first += p
    for _ in "kv":
        x = torch.randn(n_pages, hk, page, d, generator=gen, device="cuda").to(torch.float8_e4m3fn if bits8 else torch.bfloat16)
        scales = torch.randint(125, 130, (n_pages, hk, page), generator=gen, device="cuda", dtype=torch.uint8)
        value = x.double() * torch.exp2(scales.double() - 127)[..., None] if bits8 else x.double()
        mine, spoil = [], torch.ones(n_pages, page, dtype=torch.bool, device="cuda")
        for s, n in enumerate(rows):
            j = torch.arange(n, device="cuda")
            at = table[s].long()[j // page], j % page
            spoil[at] = False
            mine.append(value[at[0], :, at[1]])
        spoil = spoil[:, None].expand(-1, hk, -1)
        x.view(torch.uint8 if bits8 else torch.int16)[spoil] = 0x7F if bits8 else -1
        scales[spoil] = 255
        pool.append((x, scales))
        held.append(mine)
    return pool, table, held


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("name", PROMPTS)
def test_prompts(gpu, name, bits8):
    import torch
    new, behind, hq, hk, d, page, window, sinks, least, slices = PROMPTS[name]
    t, total = sum(new), sum(new) + 21
    rows = [a + b for a, b in zip(new, behind)]
    groups = (total * (hq // hk) // 128 + len(new)) * hk
    cfg = gpu.heads_config(hq, hk, d, norm=False, rot_dim=0)
    size = getattr(gpu.load(), "proxy_paged_quant_workspace_size" if bits8 else "proxy_paged_workspace_size")
    need = size(cfg, len(new), total, True, max(new), max(rows), window, sinks)
    cut = total * hq * slices * (4 * d + 8)
    assert groups * slices >= least and need == (0 if slices == 1 else -(-cut // 256) * 256)
    pool, table, held = filled(rows, hk, d, page, bits8, 2)
    kv_len = torch.tensor(rows, dtype=torch.int32, device="cuda")
    if bits8:
        cache = gpu.PagedCache8(cfg, {}, pool[0][0], pool[1][0], pool[0][1], pool[1][1], table, kv_len)
    else:
        cache = gpu.PagedCache(cfg, {}, pool[0][0], pool[1][0], table, kv_len)
    torch.manual_seed(3)
    q = torch.randn(total, hq, d, device="cuda").to(torch.bfloat16)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    lse = torch.full((total, hq), 5.0, device="cuda")
    out = cache.attend(q, max(rows), cu_tokens=cu, max_new=max(new), window=window, sinks=sinks, lse=lse)
    torch.cuda.synchronize()
    assert torch.isnan(out[t:]).all() and (lse[t:] == 5).all()
    n, at = max(rows), 0
    for s, (count, behind_) in enumerate(zip(new, behind)):
        for h in range(hq if count else 0):
            kv = h * hk // hq
            _, o, l, err, mag = attention64(q[at:at + count, h].double(), held[0][s][:, kv], held[1][s][:, kv], behind_,
                                            d ** -0.5, window, sinks)
            e = (d + 10) * E * err + 8 * E
            within(out[at:at + count, h], o, U["bf16"] * o.abs() + (2 * e + (n + 64) * E + 2.0 ** -8)[:, None] * mag, (name, s, h))
            within(lse[at:at + count, h], l, 2 * e + (n + 64) * E + 4 * E * l.abs(), (name, "lse", s, h))
        at += count


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hk, d", [(2, 64), (1, 128), (16, 64), (8, 128)])
def test_a_large_read(gpu, dtype, hk, d):
    """More than 65,536 tokens of few heads (a wave takes four of them) and many (one):
    long sequences between thousands of none to five rows, rows before 0, entries that
    are no page, tokens behind the last sequence; the values bit for bit."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    rng = np.random.default_rng(4)
    page, some = 16, 1500
    news = np.concatenate([[20011], rng.integers(0, 6, some), [20003], rng.integers(0, 6, some), [21002]])
    lens = news.copy()
    lens[5:some:7] -= 2  # rows before 0
    lens[9:some:7] += 3  # rows that are there already
    t, total = int(news.sum()), int(news.sum()) + 37
    assert t > 65536 and total % 16 not in (0, 4, 8, 12)
    pages = np.maximum(-(-lens // page), 1)
    n_pages = int(pages.sum()) + 5
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    first = torch.from_numpy(np.cumsum(pages) - pages).cuda()
    col = torch.arange(int(pages.max()), device="cuda")[None]
    table = torch.where(col < torch.from_numpy(pages).cuda()[:, None], order[(first[:, None] + col).clamp(max=n_pages - 1)], -1)
    table[0, 77], table[some + 1, 3], table[20, 0] = n_pages, -9, 2 ** 31 - 1
    codes = [torch.randint(0, 256, (n_pages, hk, page, d), generator=gen, device="cuda", dtype=torch.uint8) for _ in "kv"]
    scales = [torch.randint(100, 150, (n_pages, hk, page), generator=gen, device="cuda", dtype=torch.uint8) for _ in "kv"]
    cfg = gpu.heads_config(hk, hk, d, dtype=dtype, norm=False, rot_dim=0)
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = gpu.PagedCache8(cfg, {}, *(c.view(torch.float8_e4m3fn) for c in codes), *scales, table,
                            torch.tensor(lens.tolist(), **i32))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(news)]).tolist(), **i32)
    back = [torch.full((total, hk, d), 5.0, dtype=torch_dtype(dtype), device="cuda") for _ in "kv"]
    cache.read(*back, cu_tokens=cu)
    tok = torch.arange(t, device="cuda")
    seq = torch.searchsorted(cu[1:].long(), tok, right=True)
    row = torch.tensor(lens.tolist(), device="cuda")[seq] - cu.long()[seq + 1] + tok
    ids = table.long()[seq, row.clamp(min=0) // page]
    there = (row >= 0) & (ids >= 0) & (ids < n_pages)
    assert 40 < int((~there).sum()) < 2000
    at = torch.where(there, ids, 0), row.clamp(min=0) % page
    for got, c, s in zip(back, codes, scales):
        value = c[at[0], :, at[1]].view(torch.float8_e4m3fn).double() * torch.exp2(s[at[0], :, at[1]].double() - 127)[..., None]
        want = torch.where(there[:, None, None], value, 5.0).to(got.dtype)
        assert torch.equal(torch.isnan(got[:t]), torch.isnan(want))
        assert torch.equal(got[:t].nan_to_num(0.0), want.nan_to_num(0.0))
        assert (got[t:] == 5).all()
