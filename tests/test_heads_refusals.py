"""More refusals of the heads entry points: outputs on the small buffers that a
call reads. Every call here fails on the host before a launch."""
import pytest

from paper_2608_23463_amd import binding as B
from test_heads_abi import P, append, backward, cache, cfg, forward, refused, rows, weights

FAR = 64 * P
SMALL = {"gamma_q": dict(gq=FAR), "gamma_k": dict(gk=FAR), "freqs": dict(fr=FAR)}


@pytest.mark.parametrize("at", [FAR, FAR - 1024, FAR + 64], ids=["same", "from_below", "inside"])
@pytest.mark.parametrize("which", SMALL)
def test_rows_on_gains_and_frequencies(which, at):
    w = weights(**SMALL[which])
    refused(forward(w=w, qo=rows(at)))
    refused(forward(w=w, ko=rows(at)))
    refused(append(w=w, qo=rows(at)))
    refused(append(w=w, ca=cache(k_pages=at)))
    refused(append(w=w, ca=cache(v_pages=at)))
    for out in (dict(dq=rows(at)), dict(dk=rows(at))):
        refused(backward_with(w, **out))


def backward_with(w, dq=None, dk=None, pos=P):
    return B.load().proxy_qk_norm_rope_backward(cfg(), w, 5, rows(), rows(2 * P), pos, rows(3 * P), rows(4 * P),
                                                dq or rows(8 * P), dk or rows(9 * P), 5 * P, 6 * P, 7 * P, 1 << 19, None)


def test_rows_on_positions():
    for pos in (FAR, FAR + 16, FAR + 2048):  # the rows end 3 KB on, or later
        refused(forward(pos=pos, qo=rows(FAR)))
        refused(forward(pos=pos, ko=rows(FAR)))
        refused(backward(pos=pos, dq=rows(FAR)))
        refused(backward(pos=pos, dk=rows(FAR)))
        refused(append(pos=pos, qo=rows(FAR)))
        refused(append(pos=pos, ca=cache(k_pages=FAR)))


def test_append_on_its_tables():
    for name in ("page_table", "kv_len"):
        refused(append(ca=cache(**{name: 4 * P + 16})))   # q_out
        refused(append(ca=cache(**{name: 16 * P + 4096})))  # the keys' pages
        refused(append(ca=cache(**{name: 32 * P})))
    refused(append(cu=4 * P + 64))
    refused(append(cu=16 * P + 64))
    refused(append(cu=32 * P + 64))


def test_rows_side_by_side_that_meet():
    """Heads whose rows lie three side by side: a step of less than a row meets
    its neighbour, as does one that comes round to another head or token."""
    c = cfg(n_heads=8, n_kv_heads=8)
    side = lambda at, ts=8 * 192: rows(FAR + 2 * at, ts, 192)  # noqa: E731
    for at in (0, 32, -32, 56, 192 + 8, 2 * 192, 7 * 192, 8 * 192, 8 * 192 + 32, -3 * 8 * 192 + 8):
        refused(forward(c, q=side(0), qo=side(0), k=rows(2 * P), ko=side(at)))
        refused(forward(c, q=side(0), qo=rows(3 * P, 8 * 64), k=rows(2 * P), ko=side(at)))
    # tokens closer than a row (read only) count as meeting
    refused(forward(c, q=rows(FAR, 8, 192), qo=rows(3 * P), k=rows(2 * P), ko=rows(FAR + 2 * 64, 8 * 192, 192)))


def test_scales_past_the_largest():
    """The kernels take the scale times log2(e), which is infinite from 2.4e38 on."""
    from test_heads_abi import attend
    for scale in (2.4e38, -2.4e38, 3.4e38):
        refused(attend(scale=scale))
