"""Refusals of the heads entry points (norm and rotation, paged cache): every
call here fails on the host before a launch, so none needs a GPU."""
import ctypes

import pytest

from paper_2608_23463_amd import binding as B

P = 1 << 20  # a pointer that is never followed


def cfg(**kw):
    base = dict(n_heads=8, n_kv_heads=2, head_dim=64)
    base.update(kw)
    return B.heads_config(**base)


def rows(p=P, ts=512, hs=64):
    return B.PfRows(p, ts, hs)


def weights(gq=P, gk=P, fr=P):
    return B.PfHeadsWeights(gq, gk, fr)


def forward(c=None, w=None, n=5, q=None, k=None, pos=P, qo=None, ko=None):
    return B.load().proxy_qk_norm_rope_forward(c or cfg(), w or weights(), n, q or rows(), k or rows(2 * P), pos,
                                               qo or rows(3 * P), ko or rows(4 * P), None)


def backward(c=None, n=5, q=None, k=None, pos=P, dqo=None, dko=None, dq=None, dk=None, gq=5 * P, gk=6 * P, ws=7 * P,
             ws_bytes=1 << 19):
    return B.load().proxy_qk_norm_rope_backward(c or cfg(), weights(), n, q or rows(), k or rows(2 * P), pos,
                                                dqo or rows(3 * P), dko or rows(4 * P), dq or rows(8 * P),
                                                dk or rows(9 * P), gq, gk, ws, ws_bytes, None)


CACHE = dict(k_pages=16 * P, v_pages=32 * P, n_pages=10, page_size=32, page_table=P, max_pages=4, kv_len=2 * P, batch=3)


def cache(**kw):
    return B.PfPagedCache(**dict(CACHE, **kw))


def append(c=None, ca=None, n=3, cu=None, q=None, k=None, v=None, pos=None, qo=None, w=None):
    return B.load().proxy_paged_append(c or cfg(), w or weights(), ca or cache(), n, cu, q or rows(), k or rows(2 * P),
                                       v or rows(3 * P), pos, qo or rows(4 * P), None)


def attend(c=None, ca=None, n=3, cu=None, q=None, max_new=1, max_kv=100, window=0, sinks=0, scale=0.1, out=5 * P,
           lse=None, ws=6 * P, ws_bytes=1 << 30):
    return B.load().proxy_paged_attention(c or cfg(), ca or cache(), n, cu, q or rows(), max_new, max_kv, window, sinks,
                                          scale, out, lse, ws, ws_bytes, None)


def refused(status, want=B.PF_ERR_INVALID_ARG):
    assert status == want, (status, B.last_error())
    assert B.last_error()


@pytest.mark.parametrize("bad", [
    dict(n_heads=0), dict(n_kv_heads=0), dict(n_kv_heads=3), dict(rot_dim=8), dict(rot_dim=80), dict(rot_dim=-16),
    dict(style=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(axis_pairs=(16, 15)),
    dict(axis_pairs=(-1, 33)), dict(axis_pairs=(2**31 - 1, 2**31 - 1, 34)),
], ids=str)
def test_bad_configs(bad):
    for call in (forward, backward, append, attend):
        refused(call(cfg(**bad)))
    assert B.load().proxy_qk_workspace_size(cfg(**bad), 5) == 0
    assert B.load().proxy_paged_workspace_size(cfg(**bad), 3, 3, 0, 1, 1 << 20, 0, 0) == 0


def test_unsupported_configs():
    for bad in (cfg(head_dim=96), cfg(head_dim=256), cfg(n_heads=8192, n_kv_heads=2)):
        for call in (forward, backward, append, attend):
            refused(call(bad), B.PF_ERR_UNSUPPORTED)
    for field in ("dtype", "norm", "n_axes"):
        for v in (-1, 7):
            c = cfg()
            setattr(c, field, v)
            for call in (forward, backward, append, attend):
                refused(call(c))
    with pytest.raises(ValueError):
        cfg(dtype="fp16")
    with pytest.raises(ValueError):
        cfg(axis_pairs=(8, 8, 8, 8))


def test_bad_rows():
    bad = [rows(None), rows(P + 8), rows(ts=-512), rows(hs=-64), rows(ts=508), rows(hs=68), rows(ts=1 << 60), rows(hs=1 << 60)]
    for r in bad:
        refused(forward(q=r))
        refused(forward(k=r))
        refused(forward(qo=r))
        refused(forward(ko=r))
        refused(backward(q=r))
        refused(backward(dqo=r))
        refused(backward(dko=r))
        refused(backward(dq=r))
        refused(backward(dk=r))
        refused(append(k=r))
        refused(append(v=r))
        refused(append(qo=r))
        refused(attend(q=r))
        if r.p:
            refused(append(q=r))
    # rows that a call writes must not share elements; rows it reads may
    for r in (rows(ts=0), rows(hs=0), rows(ts=448, hs=64), rows(ts=64, hs=256)):
        refused(forward(qo=r))
        refused(backward(dq=r))
        refused(append(qo=r))


def test_pointers_and_counts():
    refused(forward(w=weights(fr=None)))
    refused(forward(w=weights(gq=P + 2)))
    refused(forward(w=weights(fr=P + 4)))
    refused(forward(pos=None))
    refused(forward(pos=P + 2))
    refused(forward(n=-1))
    refused(forward(n=1 << 26), B.PF_ERR_UNSUPPORTED)
    refused(backward(n=1 << 26), B.PF_ERR_UNSUPPORTED)
    refused(backward(pos=None))
    refused(backward(gq=5 * P + 2))
    refused(backward(ws=None), B.PF_ERR_WORKSPACE)
    refused(backward(ws_bytes=B.load().proxy_qk_workspace_size(cfg(), 5) - 1), B.PF_ERR_WORKSPACE)
    refused(backward(ws=7 * P + 8))
    assert forward(n=0) == append(n=0, cu=P) == attend(n=0, cu=P) == B.PF_OK  # nothing to do
    none = cfg(norm=False)
    assert B.load().proxy_qk_workspace_size(none, 5) == 0 and B.load().proxy_qk_workspace_size(cfg(), 5) >= 512
    assert B.load().proxy_qk_workspace_size(cfg(), -1) == 0


def test_overlaps():
    refused(forward(qo=rows(P + 16 * 64)))            # shifted against its input
    refused(forward(qo=rows(2 * P, 512, 64)))         # on the keys
    refused(forward(ko=rows(P)))                      # on the queries
    refused(forward(qo=rows(3 * P), ko=rows(3 * P)))
    refused(backward(dq=rows(2 * P)))                 # on the keys
    refused(backward(dq=rows(4 * P)))                 # on the keys' gradients
    refused(backward(dk=rows(3 * P)))
    refused(backward(dq=rows(8 * P), dk=rows(8 * P)))
    # bands of one fused buffer meet exactly where their columns do
    fused = lambda first: rows(P + 2 * 64 * first, 64 * 12)  # noqa: E731
    refused(forward(q=fused(0), k=fused(8), qo=fused(4), ko=rows(4 * P)))
    refused(forward(q=fused(0), k=fused(8), qo=fused(0), ko=fused(7)))
    refused(append(q=fused(0), k=fused(8), v=fused(10), qo=fused(2)))
    refused(append(k=rows(16 * P + 1024)))
    refused(append(v=rows(32 * P)))
    refused(append(qo=rows(16 * P)))
    refused(attend(out=P + 512))


def test_outputs_and_workspaces_apart():
    refused(attend(out=16 * P + 1024))                # on the pages it reads
    refused(attend(out=32 * P))
    refused(attend(lse=5 * P + 64))                   # on out
    refused(attend(lse=P + 16))                       # on the queries
    refused(attend(lse=32 * P + 16))                  # on the pages
    need = B.load().proxy_paged_workspace_size(cfg(), 3, 3, 0, 1, 4000, 0, 0)
    assert 0 < need < 8 * P
    for ws in (P, 5 * P, 16 * P, 64 * P - 256):       # queries, out, pages, lse
        refused(attend(max_kv=4000, ws=ws, lse=64 * P))
    refused(attend(max_kv=4000, ca=cache(page_table=6 * P + 16)))
    refused(attend(max_kv=4000, ca=cache(kv_len=6 * P + 16)))
    for at in (P, 2 * P, 3 * P, 4 * P, 8 * P, 9 * P):  # any rows of the call
        refused(backward(gq=at + 64))
        refused(backward(gk=at + 64))
        refused(backward(ws=at))
    refused(backward(gq=5 * P, gk=5 * P + 128))
    refused(backward(gq=7 * P))                       # on the workspace
    refused(backward(gk=7 * P + 16))


@pytest.mark.parametrize("bad", [
    dict(k_pages=None), dict(v_pages=None), dict(page_table=None), dict(kv_len=None), dict(k_pages=16 * P + 8),
    dict(page_table=P + 2), dict(kv_len=P + 1), dict(batch=0), dict(n_pages=0), dict(max_pages=0), dict(page_size=0),
    dict(page_size=-16), dict(v_pages=16 * P + 4096),
], ids=str)
def test_bad_caches(bad):
    refused(append(ca=cache(**bad)))
    refused(attend(ca=cache(**bad)))


def test_unsupported_caches():
    for bad in (dict(page_size=24), dict(max_pages=1 << 26), dict(n_pages=1 << 30), dict(page_size=2**31 - 16, max_pages=1)):
        refused(append(ca=cache(**bad)), B.PF_ERR_UNSUPPORTED)
        refused(attend(ca=cache(**bad)), B.PF_ERR_UNSUPPORTED)


def test_paged_arguments():
    refused(append(n=4))          # one token of every sequence is three
    refused(attend(n=2))
    refused(append(n=-1, cu=P))
    refused(attend(n=-1, cu=P))
    refused(append(cu=P + 2))
    refused(attend(cu=P + 2))
    refused(append(pos=P + 2))
    refused(append(n=1 << 26, cu=P), B.PF_ERR_UNSUPPORTED)
    refused(attend(n=1 << 25, cu=P), B.PF_ERR_UNSUPPORTED)
    refused(attend(n=1 << 29, cu=P), B.PF_ERR_UNSUPPORTED)
    for bad in (dict(max_new=0), dict(max_kv=0), dict(window=-1), dict(sinks=-1), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(out=None), dict(out=5 * P + 8), dict(lse=P + 2), dict(ws=6 * P + 4)):
        refused(attend(**bad))
    lib = B.load()
    need = lib.proxy_paged_workspace_size(cfg(), 3, 3, 0, 1, 1 << 20, 0, 0)
    assert need > 0 and need % 256 == 0
    refused(attend(max_kv=1 << 20, ws=None), B.PF_ERR_WORKSPACE)
    refused(attend(max_kv=1 << 20, ws_bytes=need - 1), B.PF_ERR_WORKSPACE)
    for bad in ((0, 3, 0, 1, 9, 0, 0), (3, 0, 0, 1, 9, 0, 0), (3, 3, 0, 0, 9, 0, 0), (3, 3, 0, 1, 0, 0, 0),
                (3, 3, 0, 1, 9, -1, 0), (3, 3, 0, 1, 9, 0, -1), (3, 1 << 31, 1, 1, 9, 0, 0)):
        assert lib.proxy_paged_workspace_size(cfg(), *bad) == 0
    # the largest numbers neither overflow nor refuse the query
    assert lib.proxy_paged_workspace_size(cfg(), 3, 3, 0, 2**62, 2**62, 2**62, 2**62) >= 0


def test_binding_refuses_what_is_not_on_a_gpu():
    import torch
    c = cfg(dtype="fp32")
    q, k = torch.zeros(3, 8, 64), torch.zeros(3, 2, 64)
    with pytest.raises(ValueError):
        B.qk_norm_rope_forward(c, {}, q, k, torch.zeros(1, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.qk_norm_rope_backward(c, {}, q, k, torch.zeros(1, 3, dtype=torch.int32), q, k)
    with pytest.raises(ValueError):
        B.PagedCache(c, {}, torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64), torch.zeros(3, 2, dtype=torch.int32),
                     torch.zeros(3, dtype=torch.int32))


def test_binding_refuses_other_workspaces():
    import torch
    here = torch.device("meta")
    ws = torch.empty(64, dtype=torch.uint8, device="meta")
    assert B._workspace(ws, here)[1] == 64 and B._workspace(ws.view(torch.float32), here)[1] == 64
    assert B._workspace(None, here) == (None, 0)
    for bad in (torch.empty(64, dtype=torch.uint8), ws[::2]):  # elsewhere; with gaps that are not the caller's to give
        with pytest.raises(ValueError):
            B._workspace(bad, here)


def test_rope_freqs():
    import torch
    f = B.rope_freqs(cfg(), device="cpu")
    assert f.dtype == torch.float64 and f.shape == (32,) and f[0] == 1 and torch.isclose(f[16], torch.tensor(0.01).double())
    f = B.rope_freqs(cfg(rot_dim=32, axis_pairs=(4, 4, 8)), base=100.0, device="cpu")
    assert f.shape == (16,) and f[0] == f[4] == f[8] == 1 and torch.isclose(f[6], torch.tensor(0.1).double())
    assert B.rope_freqs(cfg(rot_dim=0), device="cpu").shape == (0,)
    assert ctypes.sizeof(B.PfRows) == 24 and ctypes.sizeof(B.PfPagedCache) == 56
