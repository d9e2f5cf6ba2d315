"""Attention over whole prompts with its gradients, and a cache of 8 bits, as
measurable calls.

A case is a dict of plain values. `op` says which operator a pass calls:

  forward   binding.packed_attention_forward: causal attention over sequences
            that lie one after another, in training or for whole prompts
  backward  binding.packed_attention_backward: its gradients
  append    binding.PagedCache8.append: new tokens' keys and values into pages
            of 8-bit floating point, a power-of-two scale for every row of a
            head; what they then stand for comes back through .read
  read      binding.PagedCache8.read: rows of the pages in the rows' own type
  attend    binding.PagedCache8.attend: new tokens, one of every sequence or a
            prompt, over those pages

`own` chooses between the framework's kernels and the operators' plain form
in elementary torch operations. Head layouts are those of synth.py's workloads
(16 x 64, 8 x 64, 16 x 128) and generic ones with shared keys and values.
"""
import math
import random

import torch

own = False

EPS = 1e-6
BASE = 10000.0
TOP = 448.0  # the largest e4m3 value
LEAST = -110  # the smallest exponent of a scale


def _case(name, op, heads, kv, dim, dtype="bf16", **kw):
    return dict({"name": name} if name else {}, op=op, heads=heads, kv=kv, dim=dim, dtype=dtype, **kw)


def _packed(name, op, heads, kv, dim, batch, most, window=0, sinks=0, lens=0, **kw):
    return _case(name, op, heads, kv, dim, batch=batch, most=most, window=window, sinks=sinks, lens=lens, **kw)


def _paged(name, op, heads, kv, dim, batch, new, cached, page, ragged=False, lens=0, window=0, sinks=0, norm=False, **kw):
    return _case(name, op, heads, kv, dim, batch=batch, new=new, cached=cached, page=page, ragged=ragged, lens=lens,
                 window=window, sinks=sinks, norm=norm, **kw)


def listed():
    return [
        # one long prompt, keys shared by four query heads
        _packed("forward_prompt_8k", "forward", 32, 8, 128, 1, 8192),
        # a training batch of a windowed layer, documents packed one after another
        _packed("forward_packed_window", "forward", 16, 16, 64, 20, 2500, 600, 4, lens=1),
        # the training step's way back through packed documents, shared keys
        _packed("backward_packed_gqa", "backward", 32, 8, 128, 8, 4096, lens=2),
        # one long document of the 16 x 64 layer
        _packed("backward_8k", "backward", 16, 16, 64, 1, 8192),
        # a small windowed batch in single precision
        _packed("backward_small_fp32", "backward", 8, 2, 64, 7, 500, 100, 4, lens=3, dtype="fp32"),
        # one serving step: a token of each of 32 sequences
        _paged("append_32_tokens", "append", 16, 16, 64, 32, 1, 480, 64, True, 4),
        # prompts of many lengths taken in together, keys and queries normed and turned
        _paged("append_prompts", "append", 32, 8, 128, 24, 2600, 700, 16, True, 5, norm=True),
        # a short sequence handed over to another batch: the smallest call
        _paged("read_1_short", "read", 8, 8, 64, 1, 150, 0, 16),
        # sequences of many lengths brought back into the rows' type
        _paged("read_24_ragged", "read", 32, 8, 128, 24, 7000, 0, 64, True, 6),
        # batch serving against long caches, the repository's decode workload
        _paged("attend_32_16k", "attend", 16, 16, 64, 32, 1, 16383, 64),
        # continuous batching: sequences of many lengths, a slot or two empty
        _paged("attend_ragged_gqa", "attend", 32, 8, 128, 48, 1, 9000, 16, True, 7),
        # prompts that go on behind what is cached
        _paged("attend_prompts", "attend", 32, 8, 128, 5, 1800, 6000, 32, True, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["forward", "forward", "backward", "backward", "append", "read", "attend", "attend", "attend"])
        dim = rng.choice([64, 128])
        kv = rng.choice([1, 2, 3, 4, 8, 16])
        heads = kv * rng.choice([1, 1, 2, 4, 5, 8, 16])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        lens, ragged = rng.randrange(1 << 30), rng.random() < 0.7
        window = rng.choice([0, 0, _log(rng, 1, 4096)])
        sinks = rng.choice([0, 1, 4, 40]) if window else 0
        if op in ("forward", "backward"):
            # (the weight of a token that sees itself alone is one, and all its scores' gradients are zero)
            least = 1 if op == "forward" else 2
            c = _packed(None, op, heads, kv, dim, _log(rng, 1, 48), _log(rng, least, 8192),
                        max(window, least) if window else 0, sinks, lens, dtype=dtype)
        else:
            page = 16 * rng.choice([1, 1, 2, 3, 4, 8, 16])
            batch = _log(rng, 1, 128)
            if op == "append":
                new = rng.choice([1, _log(rng, 2, 16384)])
                c = _paged(None, op, heads, kv, dim, batch, new, _log(rng, 1, 4096), page, ragged, lens, dtype=dtype)
                # among few rows a value next to a border of its 8 bits, which
                # rounding the norm takes to either side, would be all there is
                c["norm"] = rng.random() < 0.7 and sum(n for _, n in _lengths(c)) * kv * dim >= 1 << 22
            elif op == "read":
                c = _paged(None, op, heads, kv, dim, batch, _log(rng, 1, 16384), _log(rng, 1, 64) - 1, page, ragged, lens,
                           dtype=dtype)
            else:
                new = rng.choice([1, 1, _log(rng, 2, 8192)])
                c = _paged(None, op, heads, kv, dim, batch, new, _log(rng, 1, 1 << 20 if new == 1 else 8192) - 1, page,
                           ragged, lens, window, sinks, dtype=dtype)
        if heads <= 64 and _fits(c):
            return c


def _fits(case):
    """Whether a case costs no more than the largest listed one of its operator,
    in bytes, in operations and in what the plain form spreads out."""
    for f in (lambda c: work(c)["bytes"], lambda c: work(c)["flops"] * (1 if c["dtype"] == "bf16" else 8), _held, _spread):
        if f(case) > max(f(c) for c in listed() if c["op"] == case["op"]):
            return False
    return True


# ---------------------------------------------------------------- sizes

def _size(case):
    return 2 if case["dtype"] == "bf16" else 4


def _lengths(case):
    """(rows with the new ones, new tokens) of every sequence; a packed batch is
    all new. In a step of one token each, a few slots of a ragged attention are
    empty, and a packed batch may hold a document of no tokens."""
    rng = random.Random(case["lens"])
    if "most" in case:
        n = [case["most"]] + [rng.randint(0, case["most"]) for _ in range(case["batch"] - 1)]
        return [(x, x) for x in n]
    single = case["new"] == 1
    n = [(case["cached"] + case["new"], case["new"])]
    while len(n) < case["batch"]:
        if not case["ragged"]:
            n.append(n[0])
        elif single and case["op"] == "attend" and rng.random() < 0.04:
            n.append((0, 1))
        else:
            new = 1 if single else rng.randint(0, case["new"])
            n.append((rng.randint(0, case["cached"]) + new, new))
    return n


def _pages(case):
    """Pages of every sequence."""
    return [-(-n // case["page"]) for n, _ in _lengths(case)]


def _tokens(case):
    return sum(new for _, new in _lengths(case))


def _seen(case):
    """(rows that any token sees, rows seen summed over the tokens) of every sequence."""
    w, s = case["window"], case["sinks"]
    out = []
    for n, new in _lengths(case):
        new = min(new, n)
        row = torch.arange(n - new, n)
        seen = row + 1 if not w else (row + 1).clamp(max=w) + (row + 1 - w).clamp(min=0, max=s)
        lo = max(0, n - new + 1 - w) if w else 0
        out.append((n - lo + min(s, lo) if new else 0, int(seen.sum())))
    return out


def _held(case):
    """Bytes of the cache behind a pass."""
    return 0 if "page" not in case else 2 * sum(_pages(case)) * case["page"] * case["kv"] * (case["dim"] + 1)


def _spread(case):
    """Scores that an attention in its plain form spreads out."""
    if "most" in case:
        return case["batch"] * case["most"] ** 2 * case["heads"]
    if case["op"] != "attend":
        return 0
    rows = case["cached"] + case["new"]
    if case["window"] and case["new"] == 1:
        rows = min(rows, case["window"] + case["sinks"])
    return case["batch"] * case["new"] * rows * max(case["heads"], case["kv"] * case["dim"] // case["new"])


def work(case):
    es, d, hq, hk, t = _size(case), case["dim"], case["heads"], case["kv"], _tokens(case)
    rows = (hq + hk) * d * es
    if case["op"] == "forward":
        pairs = sum(n for _, n in _seen(case))
        return {"bytes": t * (2 * rows + 4 * hq) + 4 * (case["batch"] + 1), "flops": 4 * pairs * hq * d}
    if case["op"] == "backward":
        pairs = sum(n for _, n in _seen(case))
        return {"bytes": t * (4 * rows + 4 * hq) + 4 * (case["batch"] + 1), "flops": 10 * pairs * hq * d}
    small = 4 * (sum(_pages(case)) + 2 * case["batch"])
    if case["op"] == "attend":
        seen = _seen(case)
        return {"bytes": 2 * sum(n for n, _ in seen) * hk * (d + 1) + 2 * t * hq * d * es + small,
                "flops": 4 * sum(n for _, n in seen) * hq * d}
    back = t * 2 * hk * (d * es + d + 1)  # rows read from the pages and written in their type
    if case["op"] == "read":
        return {"bytes": back + small, "flops": 2 * t * hk * d}
    put = t * (2 * hq * d * es + 2 * hk * (d * es + d + 1))
    return {"bytes": put + t * 2 * hk * d * es + small + (2 * d * es + 4 * d if case["norm"] else 0),
            "flops": t * ((hq + hk) * d * (7 if case["norm"] else 0) + 4 * hk * d)}


# ---------------------------------------------------------------- 8 bits

def _quantised(x):
    """(codes, scale bytes) of rows in 32 bits: the smallest power of two that
    takes the row's largest magnitude to at most TOP, e4m3 to nearest even."""
    m, e = torch.frexp(x.abs().amax(-1))  # m 2^e, 1/2 <= m < 1, and TOP is 7/8 2^9
    e = torch.where(m == 0, LEAST, e - 9 + (m > TOP / 512).to(e.dtype)).clamp(min=LEAST)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _power(e):
    """2^e in 32 bits, by its bits."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _values(codes, scales):
    return codes.float() * _power(scales.int() - 127)[..., None]


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    """Inputs from the seed; sizes and lengths go by the case alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    hq, hk, d = case["heads"], case["kv"], case["dim"]

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    def whole(n):
        return torch.tensor(n, dtype=torch.int32, device="cuda")

    lens = _lengths(case)
    st = {"case": case, "tokens": _tokens(case), "freqs": None, "gamma_q": None, "gamma_k": None}
    cu = [0]
    for _, new in lens:
        cu.append(cu[-1] + new)
    if "most" in case:
        st["cu"] = whole(cu)
        qkv = normal(st["tokens"], hq + 2 * hk, d)  # as one projection writes them
        st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        if case["op"] == "backward":
            st["out"], st["lse"] = _plain_packed(case, st)
            st["dout"] = normal(st["tokens"], hq, d)
    else:
        _prepare_paged(case, st, lens, cu, gen, normal, whole)
    if own:
        from paper_2608_23463_amd import binding as B
        st["cfg"] = B.heads_config(hq, hk, d, dtype=case["dtype"], norm=case.get("norm", False), eps=EPS,
                                   rot_dim=d if case.get("norm") else 0)
        if "table" in st:
            weights = {k: st[k] for k in ("gamma_q", "gamma_k", "freqs")}
            st["cache"] = B.PagedCache8(st["cfg"], weights, st["k_pages"], st["v_pages"], st["k_scales"], st["v_scales"],
                                        st["table"], st["kv_len"])
    return st


def _prepare_paged(case, st, lens, cu, gen, normal, whole):
    hq, hk, d, page = case["heads"], case["kv"], case["dim"], case["page"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    n_pages = sum(_pages(case)) + 3
    for x in ("k", "v"):
        codes, scales = _quantised(normal(n_pages, hk, page, d, dtype=torch.float32))
        # rows of other magnitudes, as layers and tokens have them
        scales += torch.randint(0, 3, scales.shape, generator=gen, device="cuda", dtype=torch.uint8)
        st[x + "_pages"], st[x + "_scales"] = codes, scales
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["batch"], max(_pages(case))), -1, dtype=torch.int32)
    starts = [0]
    for n in _pages(case):
        starts.append(starts[-1] + n)
    cols = torch.arange(table.shape[1])[None] + torch.tensor(starts[:-1])[:, None]
    used = torch.arange(table.shape[1])[None] < torch.tensor(_pages(case))[:, None]
    st["table"] = torch.where(used, order.cpu()[cols.clamp(max=n_pages - 1)], table).cuda()
    st["kv_len"] = whole([n for n, _ in lens])
    single = case["new"] == 1 and case["op"] != "read"
    rows = st["tokens"] if single or not case["ragged"] else -(-st["tokens"] // 64) * 64  # a padded batch
    st["cu"] = None if single else whole(cu)

    def blank(heads):
        return torch.zeros(rows, heads, d, device="cuda", dtype=dt)

    if case["op"] == "attend":
        st["q"] = normal(rows, hq, d) * 2
        st["out"] = blank(hq)
        return
    st["k_rows"], st["v_rows"] = blank(hk), blank(hk)
    if case["op"] == "append":
        qkv = normal(rows, hq + 2 * hk, d)
        st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        st["q_out"] = blank(hq)
        if case["norm"]:
            st["freqs"] = BASE ** (-torch.arange(d // 2, dtype=torch.float64, device="cuda") / (d // 2))
            st["gamma_q"], st["gamma_k"] = 1 + 0.1 * normal(d), 1 + 0.1 * normal(d)


# ---------------------------------------------------------------- a pass

def run(st):
    case = st["case"]
    if own:
        return _own(case, st)
    if case["op"] == "forward":
        return _plain_packed(case, st)
    if case["op"] == "backward":
        return _plain_packed_backward(case, st)
    if case["op"] == "append":
        return _plain_append(case, st)
    if case["op"] == "read":
        return _plain_read(case, st)
    return _plain_attend(case, st)


def _own(case, st):
    from paper_2608_23463_amd import binding as B
    if case["op"] == "forward":
        return B.packed_attention_forward(st["cfg"], st["q"], st["k"], st["v"], st["cu"], case["most"], window=case["window"],
                                          sinks=case["sinks"])
    if case["op"] == "backward":
        return B.packed_attention_backward(st["cfg"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["dout"], st["cu"],
                                           case["most"], window=case["window"], sinks=case["sinks"])
    if case["op"] == "append":
        st["cache"].append(st["k"], st["v"], q=st["q"], cu_tokens=st["cu"], q_out=st["q_out"])
        return [st["q_out"], *st["cache"].read(st["k_rows"], st["v_rows"], cu_tokens=st["cu"])]
    if case["op"] == "read":
        return st["cache"].read(st["k_rows"], st["v_rows"], cu_tokens=st["cu"])
    return st["cache"].attend(st["q"], case["cached"] + case["new"], cu_tokens=st["cu"], max_new=case["new"],
                              window=case["window"], sinks=case["sinks"], out=st["out"])


def _apart(case, st):
    """The packed tokens' places in sequences of the same length [B, L] and
    which of these are tokens; and what the i-th token sees [L, L]."""
    at = torch.arange(case["most"], device="cuda")
    cu = st["cu"].long()
    mine = cu[:-1, None] + at[None]
    real = mine < cu[1:, None]
    row = at[:, None]
    seen = at[None] <= row
    if case["window"]:
        seen &= (at[None] > row - case["window"]) | (at[None] < case["sinks"])
    return torch.where(real, mine, 0), real, seen


def _by_head(x, mine, kv):
    """Rows [T, H, D] in 32 bits as [B, Hk, H / Hk * L, D]."""
    b, n = mine.shape
    x = x[mine].float().view(b, n, kv, -1, x.shape[-1]).permute(0, 2, 3, 1, 4)
    return x.reshape(b, kv, -1, x.shape[-1])


def _together(x, real):
    """The rows of [B, Hk, H / Hk * L, D] that are tokens, [T, H, D]."""
    b, n = real.shape
    x = x.view(b, x.shape[1], -1, n, x.shape[-1]).permute(0, 3, 1, 2, 4)
    return x[real].flatten(1, 2)


def _weights(case, q, k, seen):
    """Softmax of the seen scores [B, Hk, H / Hk, L, L], and the log of its sums."""
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(case["dim"] ** -0.5)
    scores = scores.view(*q.shape[:2], -1, *seen.shape).masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(total), (top + total.log()).squeeze(-1)


def _plain_packed(case, st):
    mine, real, seen = _apart(case, st)
    q, k, v = (_by_head(st[x], mine, case["kv"]) for x in "qkv")
    p, lse = _weights(case, q, k, seen)
    out = torch.matmul(p.view(*q.shape[:3], -1), v)
    lse = _together(lse.reshape(*q.shape[:3], 1), real)[..., 0]
    return _together(out, real).to(st["q"].dtype), lse.contiguous()


def _plain_packed_backward(case, st):
    mine, real, seen = _apart(case, st)
    q, k, v, do = (_by_head(st[x], mine, case["kv"]) for x in ("q", "k", "v", "dout"))
    do = (do.unflatten(2, (-1, real.shape[1])) * real[:, None, None, :, None]).flatten(2, 3)
    p = _weights(case, q, k, seen)[0].view(*q.shape[:3], -1)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
    ds = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p).mul_(case["dim"] ** -0.5)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q)
    return [_together(x, real).to(st["q"].dtype) for x in (dq, dk, dv)]


def _places(case, st):
    """Page and slot of every new token, and its row."""
    at = torch.arange(st["tokens"], device="cuda")
    if st["cu"] is None:
        seq, pos = at, st["kv_len"].long() - 1
    else:
        cu = st["cu"].long()
        seq = torch.searchsorted(cu[1:], at, right=True)
        pos = st["kv_len"].long()[seq] - cu[seq + 1] + at
    return st["table"].long()[seq, pos // case["page"]], pos % case["page"], pos


def _norm_rope(case, x, gamma, pos, freqs):
    x = x.float()
    if not case["norm"]:
        return x
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma.float()
    angle = pos[:, None].double() * freqs
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _plain_append(case, st):
    n, (ids, slot, pos) = st["tokens"], _places(case, st)
    for x, rows in (("k", _norm_rope(case, st["k"][:n], st["gamma_k"], pos, st["freqs"])), ("v", st["v"][:n].float())):
        codes, scales = _quantised(rows)
        st[x + "_pages"].view(torch.uint8)[ids, :, slot] = codes.view(torch.uint8)
        st[x + "_scales"][ids, :, slot] = scales
    st["q_out"][:n] = _norm_rope(case, st["q"][:n], st["gamma_q"], pos, st["freqs"]).to(st["q"].dtype)
    return [st["q_out"], *_plain_read(case, st)]


def _plain_read(case, st):
    n, (ids, slot, _) = st["tokens"], _places(case, st)
    for x in ("k", "v"):
        codes = st[x + "_pages"].view(torch.uint8)[ids, :, slot].view(torch.float8_e4m3fn)
        st[x + "_rows"][:n] = _values(codes, st[x + "_scales"][ids, :, slot]).to(st[x + "_rows"].dtype)
    return st["k_rows"], st["v_rows"]


def _plain_attend(case, st):
    b, hq, hk, d, page = case["batch"], case["heads"], case["kv"], case["dim"], case["page"]
    new, longest = case["new"], case["cached"] + case["new"]
    lens = st["kv_len"].long()[:, None]
    w, s = case["window"], case["sinks"]
    if w and new == 1:  # the first rows, then the window
        first = (lens - w).clamp(min=0)
        sink = torch.arange(min(s, longest), device="cuda")[None].expand(b, -1)
        last = first + torch.arange(min(w, longest), device="cuda")[None]
        pos, real = torch.cat([sink, last], 1), torch.cat([sink < first, last < lens], 1)
    else:
        pos = torch.arange(longest, device="cuda")[None].expand(b, -1)
        real = pos < lens
    safe = torch.where(real, pos, 0)
    ids = torch.gather(st["table"].long(), 1, safe // page).clamp(min=0)
    k, v = (_values(st[x + "_pages"].view(torch.uint8)[ids, :, safe % page].view(torch.float8_e4m3fn),
                    st[x + "_scales"][ids, :, safe % page]) for x in "kv")  # [B, L, Hk, D]
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.permute(0, 2, 1, 3).contiguous()
    # the i-th token of every sequence, padded to the most new tokens
    cu = torch.arange(b + 1, device="cuda") if st["cu"] is None else st["cu"].long()
    mine = cu[:-1, None] + torch.arange(new, device="cuda")[None]
    is_token = mine < cu[1:, None]
    row = lens - (cu[1:] - cu[:-1])[:, None] + torch.arange(new, device="cuda")[None]  # [B, new]
    seen = real[:, None] & (pos[:, None] <= row[..., None])
    if w:
        seen = seen & ((pos[:, None] > row[..., None] - w) | (pos[:, None] < s))
    q = _by_head(st["q"], torch.where(is_token, mine, 0), hk)
    scores = torch.matmul(q, k).mul_(d ** -0.5).view(b, hk, hq // hk, new, -1)
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    p = scores.sub_(scores.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    p /= p.sum(-1, keepdim=True).clamp(min=1e-30)  # an empty slot stays zero
    o = torch.matmul(p.view(b, hk, -1, p.shape[-1]), v)
    st["out"][:st["tokens"]] = _together(o, is_token).to(st["q"].dtype)
    return st["out"]


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    """From the definitions in 64 bits, sequence by sequence and head by head:
    gradients by automatic differentiation, rotations as complex factors, 8 bits
    by rounding to whole steps."""
    st = prepare(case, seed)
    if case["op"] == "forward":
        out, lse = st["q"].double(), torch.empty(st["q"].shape[:2], dtype=torch.float64, device="cuda")
        for rows, h, hk in _sequence_heads(case):
            out[rows, h], lse[rows, h] = _defined(case, st["q"][rows, h].double(), st["k"][rows, hk].double(),
                                                  st["v"][rows, hk].double())
        return out, lse
    if case["op"] == "backward":
        grads = [torch.zeros(st[x].shape, dtype=torch.float64, device="cuda") for x in "qkv"]
        for rows, h, hk in _sequence_heads(case):
            leaves = [st[x][rows, i].double().requires_grad_() for x, i in (("q", h), ("k", hk), ("v", hk))]
            got = torch.autograd.grad(_defined(case, *leaves)[0], leaves, st["dout"][rows, h].double())
            for g, total, i in zip(got, grads, (h, hk, hk)):
                total[rows, i] += g
        return grads
    if case["op"] == "attend":
        return _exact_attend(case, st)
    q_out = st["q_out"].double() if case["op"] == "append" else None
    k_rows, v_rows = st["k_rows"].double(), st["v_rows"].double()
    first = 0
    for i, (n, new) in enumerate(_lengths(case)):
        rows, pos = slice(first, first + new), torch.arange(n - new, n, device="cuda")
        first += new
        if case["op"] == "append":
            q_out[rows] = _turned(case, st["q"][rows], st["gamma_q"], pos, st["freqs"])
            k_rows[rows] = _rounded(_turned(case, st["k"][rows], st["gamma_k"], pos, st["freqs"]))
            v_rows[rows] = _rounded(st["v"][rows].double())
        else:
            pages, at = st["table"][i, :-(-n // case["page"])].long(), pos % case["page"]
            k_rows[rows], v_rows[rows] = (_held_values(st, x, pages)[pos // case["page"], :, at] for x in "kv")
    return [k_rows, v_rows] if q_out is None else [q_out, k_rows, v_rows]


def _sequence_heads(case):
    first = 0
    for n, _ in _lengths(case):
        for h in range(case["heads"] if n else 0):
            yield slice(first, first + n), h, h // (case["heads"] // case["kv"])
        first += n


def _defined(case, q, k, v, first=0):
    """Attention of tokens at rows first.. over rows 0.., and the log-sums."""
    row, at = first + torch.arange(q.shape[0], device="cuda")[:, None], torch.arange(k.shape[0], device="cuda")
    hidden = at > row
    if case["window"]:
        hidden |= (at <= row - case["window"]) & (at >= case["sinks"])
    logits = ((q @ k.t()) / math.sqrt(case["dim"])).masked_fill(hidden, -math.inf)
    return torch.softmax(logits, -1) @ v, torch.logsumexp(logits, -1)


def _rounded(x):
    """What rows in 64 bits stand for once they are held in 8."""
    top = x.abs().amax(-1, keepdim=True)
    scale = _wide_power(torch.ceil(torch.log2(top / TOP)).clamp(min=LEAST).long())
    for _ in range(2):  # the logarithm may have rounded across a power of two
        scale = torch.where(top > TOP * scale, 2 * scale, torch.where((top <= TOP * scale / 2) & (scale > 2.0 ** LEAST), scale / 2, scale))
    y = x / scale
    step = _wide_power(torch.frexp(y)[1].clamp(min=-5).long() - 4)  # three bits behind the first; 2^-9 at the least
    return torch.round(y / step) * step * scale


def _turned(case, x, gamma, pos, freqs):
    x = x.double()
    if not case["norm"]:
        return x
    x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * gamma.double()
    angle = pos.double()[:, None] * freqs[None]
    c = torch.complex(x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:])
    c = c * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat([c.real, c.imag], -1)


def _wide_power(e):
    return ((e + 1023) << 52).view(torch.float64)


def _held_values(st, x, pages=slice(None)):
    """The 64-bit values of an array of 8-bit pages."""
    codes = st[x + "_pages"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).float().double()
    return codes * _wide_power(st[x + "_scales"][pages].long() - 127)[..., None]


def _exact_attend(case, st):
    out = st["out"].double()
    first = 0
    for i, (n, new) in enumerate(_lengths(case)):
        rows = slice(first, first + new)
        first += new
        if n == 0 or new == 0:
            continue
        pages = st["table"][i, :-(-n // case["page"])].long()
        k, v = (_held_values(st, x, pages) for x in "kv")
        for h in range(case["heads"]):
            hk = h // (case["heads"] // case["kv"])
            out[rows, h] = _defined(case, st["q"][rows, h].double(), k[:, hk].reshape(-1, case["dim"])[:n],
                                    v[:, hk].reshape(-1, case["dim"])[:n], n - new)[0]
    return out
