"""CPU checks: the latent cache's calls refuse bad arguments on the host, before anything reaches a GPU."""

import os

import numpy as np
import pytest

from paper_2607_20507_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

P = 0x1000  # an address that no refused call may touch
OK, INVALID, UNSUPPORTED = B.SPEC_OK, B.SPEC_E_INVALID, B.SPEC_E_UNSUPPORTED
NAN, INF = float("nan"), float("inf")


def last():
    return B.lib().spec_last_error(None).decode()


APPEND = dict(dt=1, R=4, H=8, nope=128, rope=64, rank=512, theta=1e4, eps=1e-5, q=P, kv=P, w=P, pos=P, slot=P, P=10, out=P, pages=P)


@pytest.mark.parametrize("change, status", [
    (dict(dt=2), INVALID), (dict(R=-1), INVALID), (dict(H=0), INVALID), (dict(H=65536), INVALID), (dict(theta=0.0), INVALID),
    (dict(theta=NAN), INVALID), (dict(eps=-1e-9), INVALID), (dict(eps=NAN), INVALID), (dict(P=-1), INVALID), (dict(P=(1 << 27) + 1), INVALID),
    (dict(nope=96), UNSUPPORTED), (dict(rope=128), UNSUPPORTED), (dict(rank=384), UNSUPPORTED), (dict(rank=0), UNSUPPORTED),
    (dict(q=None), INVALID), (dict(kv=None), INVALID), (dict(w=None), INVALID), (dict(pos=None), INVALID), (dict(slot=None), INVALID),
    (dict(out=None), INVALID), (dict(pages=None), INVALID), (dict(q=P + 4), INVALID), (dict(kv=P + 8), INVALID), (dict(w=P + 2), INVALID),
    (dict(out=P + 2), INVALID), (dict(pages=P + 8), INVALID), (dict(R=0), OK)])
def test_rope_latent(change, status):
    a = {**APPEND, **change}
    got = B.lib().spec_op_rope_latent(a["dt"], a["R"], a["H"], a["nope"], a["rope"], a["rank"], a["theta"], a["eps"], a["q"], a["kv"],
                                      a["w"], a["pos"], a["slot"], a["P"], a["out"], a["pages"], None)
    assert got == status
    if status != OK:
        assert "spec_op_rope_latent" in last()


ATT = dict(dt=1, n=2, rows=[1, 2], pos0=[30, 0], table=[[0, 1, 9], [2, 3, 9]], max_pages=3, P=10, H=8, nope=128, rope=64, rank=512, v=128,
           scale=0.1, q=P, pages=P, wk=P, ks=128 * 512, wv=P, vs=128 * 512, out=P, ws=P, nbytes=1 << 30)


def attention(a):
    i32 = lambda x: None if x is None else np.array(x, dtype=np.int32)  # noqa: E731
    rows, pos0, table = i32(a["rows"]), i32(a["pos0"]), i32(a["table"])
    at = lambda x: None if x is None else x.ctypes.data  # noqa: E731
    need = B.lib().spec_op_attention_latent_workspace_bytes(a["dt"], a["n"], at(rows), at(pos0), a["max_pages"], a["H"], a["nope"], a["rope"],
                                                            a["rank"], a["v"])
    got = B.lib().spec_op_attention_latent(a["dt"], a["n"], at(rows), at(pos0), at(table), a["max_pages"], a["P"], a["H"], a["nope"], a["rope"],
                                           a["rank"], a["v"], a["scale"], a["q"], a["pages"], a["wk"], a["ks"], a["wv"], a["vs"], a["out"],
                                           a["ws"], a["nbytes"] if a["nbytes"] is not None else need - 1, None)
    return got, need


@pytest.mark.parametrize("change, status, sized", [
    # sized: the workspace is still asked for
    (dict(dt=3), INVALID, False), (dict(n=-1), INVALID, False), (dict(max_pages=0), INVALID, False), (dict(H=0), INVALID, False),
    (dict(H=65536), INVALID, False), (dict(rows=None), INVALID, False), (dict(pos0=None), INVALID, False),
    (dict(rows=[-1, 2]), INVALID, False), (dict(pos0=[-1, 0]), INVALID, False), (dict(pos0=[48, 0]), INVALID, False),
    (dict(pos0=[1 << 30, 0], max_pages=1 << 27), INVALID, False), (dict(rows=[1, (1 << 27) + 1], max_pages=1 << 24), INVALID, False),
    (dict(pos0=[2147483647, 0]), INVALID, False),
    (dict(nope=32), UNSUPPORTED, False), (dict(rope=16), UNSUPPORTED, False), (dict(rank=1024), UNSUPPORTED, False), (dict(v=256), UNSUPPORTED, False),
    (dict(table=[[0, 1, 9], [10, 3, 9]]), INVALID, True), (dict(table=[[0, -1, 9], [2, 3, 9]]), INVALID, True),
    (dict(table=None), INVALID, True), (dict(scale=0.0), INVALID, True), (dict(scale=-1.0), INVALID, True), (dict(scale=NAN), INVALID, True),
    (dict(scale=INF), INVALID, True), (dict(q=None), INVALID, True), (dict(pages=None), INVALID, True), (dict(wk=None), INVALID, True),
    (dict(wv=None), INVALID, True), (dict(out=None), INVALID, True), (dict(ws=None), INVALID, True), (dict(q=P + 8), INVALID, True),
    (dict(pages=P + 8), INVALID, True), (dict(wk=P + 2), INVALID, True), (dict(wv=P + 2), INVALID, True), (dict(out=P + 4), INVALID, True),
    (dict(ws=P + 16), INVALID, True), (dict(ks=128 * 512 - 8), INVALID, True), (dict(vs=128 * 512 + 4), INVALID, True),
    (dict(vs=-128 * 512), INVALID, True), (dict(ks=1 << 41), INVALID, True), (dict(nbytes=None), INVALID, True), (dict(nbytes=0), INVALID, True),
    (dict(rows=[0, 0]), OK, False), (dict(n=0), OK, False)])
def test_attention_latent(change, status, sized):
    got, need = attention({**ATT, **change})
    assert got == status and (need > 0) == sized
    if status != OK:
        assert "spec_op_attention_latent" in last()


def test_a_page_that_no_row_needs_is_not_looked_at():
    """Entries behind a sequence's last page, and a whole row of a sequence without rows, may hold anything; here the next refusal is
    the scale's or the buffers', not theirs."""
    got, _ = attention({**ATT, "rows": [0, 2], "table": [[-5, 99, 99], [2, -1, 77]], "ws": P + 16})
    assert got == INVALID and "aligned" in last()
