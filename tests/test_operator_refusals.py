"""CPU checks: the calls of the token scores, the cache pages and the 4-bit
cache refuse bad arguments on the host, before anything reaches a GPU."""

import os

import numpy as np
import pytest

from paper_2607_20507_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

P = 0x1000  # an address that no refused call may touch
OK, INVALID, UNSUPPORTED = B.SPEC_OK, B.SPEC_E_INVALID, B.SPEC_E_UNSUPPORTED


def i32(*v):
    return np.array(v, dtype=np.int32)


def last():
    return B.lib().spec_last_error(None).decode()


SCORE = dict(rows=2, V=100, logits=P, ld=100, temps=P, tokens=P, n_top=4, logp=P, ent=P, ids=P, top=P, ws=P, nbytes=1 << 20)


@pytest.mark.parametrize("change, status", [
    (dict(rows=-1), INVALID), (dict(V=0), INVALID), (dict(ld=99), INVALID), (dict(n_top=-1), INVALID),
    (dict(n_top=65, V=100), INVALID), (dict(n_top=5, V=4), INVALID), (dict(logits=None), INVALID), (dict(ws=None), INVALID),
    (dict(tokens=None), INVALID), (dict(ids=None), INVALID), (dict(top=None), INVALID), (dict(logits=P + 2), INVALID),
    (dict(ws=P + 8), INVALID), (dict(nbytes=63), INVALID), (dict(rows=0), OK)])
def test_token_logprobs(change, status):
    a = {**SCORE, **change}
    got = B.lib().spec_token_logprobs(a["rows"], a["V"], a["logits"], a["ld"], a["temps"], a["tokens"], a["n_top"], a["logp"],
                                      a["ent"], a["ids"], a["top"], a["ws"], a["nbytes"], None)
    assert got == status
    if status != OK:
        assert "spec_token_logprobs" in last()


def test_logprobs_workspace():
    f = B.lib().spec_token_logprobs_workspace_bytes
    assert f(0, 100, 1) == 0 and f(1, 0, 1) == 0 and f(1, 100, 65) == 0 and f(1, 100, -1) == 0
    assert f(8, 32000, 0) > 0 and f(8, 32000, 64) > f(8, 32000, 0)


@pytest.mark.parametrize("src, dst, change, status", [
    ((1, 2), (3, 3), {}, INVALID),            # a destination twice
    ((1, 2), (2, 3), {}, INVALID),            # a destination that is a source
    ((4,), (4,), {}, INVALID),                # onto itself
    ((-1,), (3,), {}, INVALID), ((8,), (3,), {}, INVALID), ((1,), (8,), {}, INVALID), ((1,), (-1,), {}, INVALID),
    ((1,), (2,), dict(page=0), UNSUPPORTED), ((1,), (2,), dict(page=24), UNSUPPORTED),
    ((1,), (2,), dict(planes=65536), UNSUPPORTED), ((1,), (2,), dict(planes=-1), INVALID), ((1,), (2,), dict(pages=-1), INVALID),
    ((1,), (2,), dict(pool=None), INVALID), ((1,), (2,), dict(pool=P + 8), INVALID), ((1,), (2,), dict(ws=None), INVALID),
    ((1,), (2,), dict(nbytes=0), INVALID), ((), (), {}, OK), ((1,), (2,), dict(planes=0), OK)])
def test_copy_pages(src, dst, change, status):
    a = {**dict(planes=2, pages=8, page=64, pool=P, ws=P, nbytes=1 << 16), **change}
    s, d = i32(*src), i32(*dst)
    assert B.lib().spec_op_kv_copy_pages(a["planes"], a["pages"], a["page"], a["pool"], len(s), s.ctypes.data, d.ctypes.data,
                                         a["ws"], a["nbytes"], None) == status


ROPE = dict(dtype=1, R=4, hq=8, hkv=2, hd=128, theta=1e4, qkv=P, pos=P, slot=P, pages=8, q=P, k=P, v=P)


@pytest.mark.parametrize("change, status", [
    (dict(dtype=2), INVALID), (dict(R=-1), INVALID), (dict(hq=0), INVALID), (dict(hkv=0), INVALID), (dict(theta=0.0), INVALID),
    (dict(theta=float("nan")), INVALID), (dict(pages=-1), INVALID), (dict(pages=1 << 30), INVALID), (dict(hd=96), UNSUPPORTED),
    (dict(hd=256), UNSUPPORTED), (dict(qkv=None), INVALID), (dict(pos=None), INVALID), (dict(slot=None), INVALID),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(qkv=P + 4), INVALID), (dict(q=P + 8), INVALID),
    (dict(k=P + 4), INVALID), (dict(R=0), OK)])
def test_rope_kv4(change, status):
    a = {**ROPE, **change}
    assert B.lib().spec_op_rope_kv4(a["dtype"], a["R"], a["hq"], a["hkv"], a["hd"], a["theta"], a["qkv"], a["pos"], a["slot"],
                                    a["pages"], a["q"], a["k"], a["v"], None) == status


@pytest.mark.parametrize("change, status", [
    (dict(dtype=-1), INVALID), (dict(R=-1), INVALID), (dict(hkv=0), INVALID), (dict(pages=-2), INVALID), (dict(hd=32), UNSUPPORTED),
    (dict(slot=None), INVALID), (dict(k=None), INVALID), (dict(ko=None), INVALID), (dict(vo=P + 2), INVALID), (dict(R=0), OK),
    (dict(pages=0), OK)])
def test_kv4_read(change, status):
    a = {**dict(dtype=0, R=4, hkv=2, hd=64, slot=P, pages=8, k=P, v=P, ko=P, vo=P), **change}
    assert B.lib().spec_op_kv4_read(a["dtype"], a["R"], a["hkv"], a["hd"], a["slot"], a["pages"], a["k"], a["v"], a["ko"], a["vo"],
                                    None) == status


ATTN = dict(dtype=1, rows=(2, 3), pos0=(10, 0), table=((0, 1), (2, 3)), pages=4, hq=8, hkv=2, hd=128, q=P, k=P, v=P, o=P, ws=P,
            nbytes=1 << 40)


@pytest.mark.parametrize("change, status", [
    (dict(dtype=3), INVALID), (dict(hq=9), INVALID), (dict(hkv=0), INVALID), (dict(hd=80), UNSUPPORTED), (dict(hq=130), UNSUPPORTED),
    (dict(dtype=0, hq=66), UNSUPPORTED), (dict(rows=(-1, 3)), INVALID), (dict(pos0=(-1, 0)), INVALID), (dict(pos0=(31, 0)), INVALID),
    (dict(pos0=(2 ** 31 - 1, 0)), INVALID), (dict(table=((0, 4), (2, 3))), OK), (dict(table=((4, 1), (2, 3))), INVALID),
    (dict(table=((-1, 1), (2, 3))), INVALID), (dict(q=None), INVALID), (dict(o=None), INVALID), (dict(ws=None), INVALID),
    (dict(ws=P + 16), INVALID), (dict(nbytes=100), INVALID), (dict(rows=(0, 0)), OK), (dict(pages=0), INVALID)])
def test_attention_kv4(change, status):
    a = {**ATTN, **change}
    if status == OK and "table" in change:
        a["rows"] = (0, 0)  # a page id that no row needs is not looked at
    r, p, t = i32(*a["rows"]), i32(*a["pos0"]), np.array(a["table"], dtype=np.int32)
    got = B.lib().spec_op_attention_kv4(a["dtype"], len(r), r.ctypes.data, p.ctypes.data, t.ctypes.data, t.shape[1], a["pages"],
                                        a["hq"], a["hkv"], a["hd"], a["q"], a["k"], a["v"], a["o"], a["ws"], a["nbytes"], None)
    assert got == status
    if status != OK:
        assert "spec_op_attention_kv4" in last()


def test_sizes_that_pass_32_bits():
    big, L = (1 << 30) + 1, B.lib()
    r, p = i32(1), i32(big - 1)
    assert L.spec_token_logprobs(1, big, P, big, P, P, 4, P, P, P, P, P, 1 << 40, None) == UNSUPPORTED and "2^30" in last()
    assert L.spec_token_logprobs_workspace_bytes(1, big, 4) == 0 and L.spec_token_logprobs_workspace_bytes(1, big - 1, 4) > 0
    assert L.spec_op_attention_kv4_workspace_bytes(1, 1, r.ctypes.data, p.ctypes.data, big, 8, 2, 128) == 0
    assert "2^30" in last()
    p = i32(big - 2)  # the longest
    assert L.spec_op_attention_kv4_workspace_bytes(1, 1, r.ctypes.data, p.ctypes.data, big, 8, 2, 128) > 4 * (big // 16)
    assert L.spec_op_rope_kv4(1, 4, 65536, 2, 128, 1e4, P, P, P, 8, P, P, P, None) == INVALID
    assert L.spec_op_rope_kv4(1, 4, 2, 65536, 128, 1e4, P, P, P, 8, P, P, P, None) == INVALID
    assert L.spec_op_kv4_read(1, 4, 65536, 128, P, 8, P, P, P, P, None) == INVALID
    assert L.spec_op_attention_kv4_workspace_bytes(1, 1, r.ctypes.data, r.ctypes.data, 1, 65536, 65536, 128) == 0


def test_attention_kv4_workspace():
    f = B.lib().spec_op_attention_kv4_workspace_bytes
    r, p = i32(6), i32(2047)
    assert f(1, 1, r.ctypes.data, p.ctypes.data, 129, 32, 8, 128) > 0
    assert f(1, 1, r.ctypes.data, p.ctypes.data, 128, 32, 8, 128) == 0  # rows beyond the table
    assert f(1, 1, None, None, 129, 32, 8, 128) == 0
    zero = i32(0)
    assert f(1, 1, zero.ctypes.data, p.ctypes.data, 129, 32, 8, 128) == 0


def test_binding_checks_tensors():
    torch = pytest.importorskip("torch")
    cpu = torch.zeros(2, 100)
    with pytest.raises(ValueError):
        B.spec_token_logprobs(cpu, None, None, None, None, None, None, cpu)
    with pytest.raises(ValueError):
        B.spec_op_kv_copy_pages(torch.zeros(2, 4, 16), [1, 2], [3], cpu)
    with pytest.raises(ValueError):
        B.spec_op_attention_kv4(1, [1], [0, 1], [[0]], 1, 8, 2, 128, cpu, cpu, cpu, cpu, cpu)
