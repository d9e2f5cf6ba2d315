"""Refusals of the packed attention and of the 8-bit cache: every call here
fails on the host before a launch, so none needs a GPU."""
import pytest

from paper_2608_23463_amd import binding as B
from test_heads_abi import CACHE, P, cfg, refused, rows, weights

FAR = 64 * P
UNSUPPORTED = B.PF_ERR_UNSUPPORTED


def forward(c=None, batch=3, n=5, cu=P, q=None, k=None, v=None, most=5, window=0, sinks=0, scale=0.1, out=5 * P, lse=6 * P):
    return B.load().proxy_packed_attention_forward(c or cfg(), batch, n, cu, q or rows(2 * P), k or rows(3 * P),
                                                   v or rows(4 * P), most, window, sinks, scale, out, lse, None)


def backward(c=None, batch=3, n=5, cu=P, q=None, k=None, v=None, most=5, window=0, sinks=0, scale=0.1, out=5 * P, lse=6 * P,
             do=None, dq=None, dk=None, dv=None, ws=11 * P, ws_bytes=1 << 19):
    return B.load().proxy_packed_attention_backward(c or cfg(), batch, n, cu, q or rows(2 * P), k or rows(3 * P),
                                                    v or rows(4 * P), most, window, sinks, scale, out, lse, do or rows(7 * P),
                                                    dq or rows(8 * P), dk or rows(9 * P), dv or rows(10 * P), ws, ws_bytes,
                                                    None)


def cache(ks=48 * P, vs=49 * P, **kw):
    return B.PfPagedQuantCache(B.PfPagedCache(**dict(CACHE, **kw)), ks, vs)


def append(c=None, ca=None, n=3, cu=None, q=None, k=None, v=None, pos=None, qo=None, w=None):
    return B.load().proxy_paged_quant_append(c or cfg(), w or weights(), ca or cache(), n, cu, q or rows(), k or rows(2 * P),
                                             v or rows(3 * P), pos, qo or rows(4 * P), None)


def read(c=None, ca=None, n=3, cu=None, k=None, v=None):
    return B.load().proxy_paged_quant_read(c or cfg(), ca or cache(), n, cu, k or rows(3 * P), v or rows(4 * P), None)


def attend(c=None, ca=None, n=3, cu=None, q=None, max_new=1, max_kv=100, window=0, sinks=0, scale=0.1, out=5 * P,
           lse=None, ws=6 * P, ws_bytes=1 << 19):
    return B.load().proxy_paged_quant_attention(c or cfg(), ca or cache(), n, cu, q or rows(), max_new, max_kv, window, sinks,
                                                scale, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_packed_arguments(call):
    for bad in (dict(batch=0), dict(n=-1), dict(cu=None), dict(cu=P + 2), dict(most=0), dict(window=-1), dict(sinks=-1),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2.4e38), dict(out=None), dict(out=5 * P + 8),
                dict(lse=None), dict(lse=6 * P + 2), dict(q=B.PfRows(None, 512, 64)), dict(k=rows(3 * P + 8)),
                dict(v=rows(4 * P, 511)), dict(q=rows(2 * P, -512)), dict(c=cfg(n_kv_heads=3))):
        refused(call(**bad))
    for bad in (dict(c=cfg(head_dim=96)), dict(n=1 << 28), dict(batch=2**31 - 1), dict(k=rows(3 * P, (1 << 23) + 8)),
                dict(v=rows(4 * P, 1 << 24))):
        refused(call(**bad), UNSUPPORTED)
    assert call(n=0, q=B.PfRows(None, 0, 0), out=None, lse=None) == 0


def test_packed_outputs_on_inputs():
    for at in (2 * P, 3 * P + 64, 4 * P + 1024, P):
        refused(forward(out=at))
        refused(forward(lse=at))
    refused(forward(out=FAR, lse=FAR + 64))
    for name in ("dq", "dk", "dv"):
        for at in (2 * P, 3 * P, 4 * P + 64, 5 * P, 6 * P, 7 * P + 512, P, 11 * P):
            refused(backward(**{name: rows(at)}))
        refused(backward(**{name: rows(FAR, 32, 64)}))  # rows on each other
    refused(backward(dq=rows(FAR), dk=rows(FAR + 64)))
    refused(backward(dk=rows(FAR), dv=rows(FAR + 64)))
    for at in (2 * P, 5 * P, 6 * P, 7 * P, 8 * P, 9 * P, 10 * P, P):
        refused(backward(ws=at))


def test_packed_workspace():
    need = B.load().proxy_packed_workspace_size(cfg(), 3, 5, 5, 0, 0)
    assert need >= 8 * 5 * 8
    refused(backward(ws_bytes=need - 1), B.PF_ERR_WORKSPACE)
    refused(backward(ws=None), B.PF_ERR_WORKSPACE)
    refused(backward(ws=11 * P + 8))
    for bad in ((cfg(head_dim=96), 3, 5), (cfg(), 0, 5), (cfg(), 3, 0), (cfg(), 3, -1), (cfg(), 3, 1 << 40)):
        assert B.load().proxy_packed_workspace_size(*bad, 5, 0, 0) == 0
    for bad in ((0, 0, 0), (5, -1, 0), (5, 0, -1)):
        assert B.load().proxy_packed_workspace_size(cfg(), 3, 5, *bad) == 0


def test_quant_cache_arguments():
    for bad in (dict(ks=None), dict(vs=None), dict(ks=48 * P + 8), dict(vs=49 * P + 1), dict(k_pages=None), dict(v_pages=P + 8),
                dict(page_table=None), dict(kv_len=None), dict(batch=0), dict(n_pages=0), dict(ks=16 * P), dict(vs=32 * P + 64),
                dict(vs=48 * P + 16), dict(k_pages=32 * P + 1024)):
        for call in (append, read, attend):
            refused(call(ca=cache(**bad)))
    for bad in (dict(page_size=24), dict(max_pages=1 << 30), dict(n_pages=1 << 30)):
        for call in (append, read, attend):
            refused(call(ca=cache(**bad)), UNSUPPORTED)
    for call in (append, read, attend):
        refused(call(n=4))
        refused(call(n=-1))
        refused(call(cu=P + 1))
        assert call(n=0, cu=P) == 0


def test_quant_outputs_on_what_is_read():
    for at in (16 * P, 32 * P + 1024, 48 * P, 49 * P + 64, P, 2 * P):  # pages, scales, table, lengths
        refused(read(k=rows(at)))
        refused(read(v=rows(at)))
        refused(append(qo=rows(at)))
        refused(attend(out=at))
        refused(attend(lse=at))
    refused(read(k=rows(FAR), v=rows(FAR + 64)))
    refused(read(k=rows(FAR, 32, 64)))
    refused(append(k=rows(48 * P)))
    refused(append(v=rows(16 * P)))
    refused(append(ca=cache(ks=FAR), qo=rows(FAR - 64)))
    refused(append(pos=FAR, ca=cache(vs=FAR)))


def test_quant_attention_arguments():
    for bad in (dict(max_new=0), dict(max_kv=0), dict(window=-1), dict(sinks=-1), dict(scale=float("nan")), dict(out=None),
                dict(out=5 * P + 8), dict(lse=6 * P + 2), dict(q=rows(P + 8))):
        refused(attend(**bad))
    need = B.load().proxy_paged_quant_workspace_size(cfg(), 3, 3, 0, 1, 100000, 0, 0)
    assert need > 0
    refused(attend(max_kv=100000, ws_bytes=need - 1), B.PF_ERR_WORKSPACE)
    assert B.load().proxy_paged_quant_workspace_size(cfg(), 0, 3, 0, 1, 100000, 0, 0) == 0
