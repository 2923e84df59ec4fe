"""Forked sequences and compacted pools on a GPU: every continuation equals the
one of a sequence that was prefilled under that id, whatever its siblings do to
the pages they share."""

import numpy as np
import pytest

from gpu_util import device, say
from workloads import SMALL_BF16, TINY_FP32, model_weights, uniform_prompts

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PAGES = 24


def models(which):
    from paper_2607_20507_amd.session import DeviceModel
    cfg, lt, ld = (TINY_FP32, None, None) if which == "fp32" else (SMALL_BF16, 2, 1)
    dev = device()
    return cfg, (DeviceModel(cfg.target, model_weights(cfg.target, cfg.seed, lt), dev, n_layers=lt),
                 DeviceModel(cfg.draft, model_weights(cfg.draft, cfg.seed + 1, ld), dev, n_layers=ld))


def session(pair, seqs=6, pages=None, draft=True):
    from paper_2607_20507_amd.session import SpecSession
    return SpecSession(pair[0], pair[1] if draft else None, max_seqs=seqs, k_max=4, max_pages_per_seq=PAGES, max_rows=256,
                       num_pages_target=pages, num_pages_draft=pages if draft else None)


def rounds(s, sid, n, seed=3, temps=0.8):
    """n speculative rounds of one sequence: accepted counts, tokens and logits of each."""
    out = []
    for r in range(n):
        s.draft_loop([sid], [temps], seed + r, [4])
        na, tok = s.verify([sid], [temps], seed + r)
        out.append((int(na[0]), tok[0].tolist(), s.last_logits().cpu().numpy()))
        s.commit([sid], na)
    return out


def same(a, b):
    assert len(a) == len(b)
    for (n1, t1, z1), (n2, t2, z2) in zip(a, b):
        assert n1 == n2 and t1 == t2 and np.array_equal(z1, z2)


def alone(pair, prompt, sid, n, before=0):
    """The rounds of a sequence in a context of its own, after `before` others."""
    s = session(pair)
    s.prefill([sid], [prompt])
    got = rounds(s, sid, before + n)[before:]
    s.close()
    return got


@pytest.mark.parametrize("which", ["fp32", "bf16"])
@pytest.mark.parametrize("length", [1, 16, 17, 49, 61])
def test_forks_continue_as_prefilled_sequences(which, length):
    cfg, pair = models(which)
    prompt = uniform_prompts(cfg.seed + 1, [length], cfg.target.vocab)[0]
    say("fork", which, length)
    s = session(pair)
    s.prefill([10], [prompt])
    s.fork(10, [11, 12])
    info = {i: s.seq_info(i) for i in (10, 11, 12)}
    full = (length - 1) // 16
    for side in ("pages_target", "pages_draft"):
        assert all(info[i][side][:full] == info[10][side][:full] for i in (11, 12))  # full pages are shared
        rest = [p for i in (10, 11, 12) for p in info[i][side][full:]]
        assert len(rest) == len(set(rest)) == (3 if (length - 1) % 16 else 0)        # the partial one is each one's own
    got = {12: rounds(s, 12, 2), 10: rounds(s, 10, 2)}  # in any order, long past the shared pages
    got[11] = rounds(s, 11, 2)
    for sid, g in got.items():
        same(g, alone(pair, prompt, sid, 2))
    s.close()


def test_fork_between_rounds_and_of_forks():
    cfg, pair = models("bf16")
    prompt = uniform_prompts(cfg.seed + 2, [37], cfg.target.vocab)[0]
    s = session(pair)
    s.prefill([5], [prompt])
    rounds(s, 5, 2)
    s.fork(5, [6])
    s.fork(6, [7])
    base = [s.seq_info(i) for i in (5, 6, 7)]
    assert len({(b["target_len"], b["draft_len"], b["pending_pos"]) for b in base}) == 1
    a = rounds(s, 7, 2, seed=50)
    s.release(5)  # the pages stay with the others
    b = rounds(s, 6, 2, seed=50)
    t = session(pair)
    t.prefill([5], [prompt])
    rounds(t, 5, 2)
    for sid, want in ((7, a), (6, b)):
        t.fork(5, [sid])
        same(rounds(t, sid, 2, seed=50), want)
        t.release(sid)
    s.close()
    t.close()


@pytest.mark.parametrize("new_len", [0, 1, 15, 16, 17, 32, 40, 47, 48])
def test_rollback_into_shared_pages(new_len):
    """A rollback of one sequence leaves the others' caches as they are, and goes on as a shorter prompt."""
    cfg, pair = models("fp32")
    prompt = uniform_prompts(cfg.seed + 3, [53], cfg.target.vocab)[0]
    s = session(pair)
    s.prefill([1], [prompt])
    s.fork(1, [2, 3])
    s.rollback(2, new_len)
    i1, i2 = s.seq_info(1), s.seq_info(2)
    assert i2["target_len"] == new_len and i2["pages_target"][:new_len // 16] == i1["pages_target"][:new_len // 16]
    if new_len % 16:
        assert i2["pages_target"][-1] not in i1["pages_target"] + s.seq_info(3)["pages_target"]
    got2 = rounds(s, 2, 2)
    same(rounds(s, 1, 2), alone(pair, prompt, 1, 2))
    same(rounds(s, 3, 2), alone(pair, prompt, 3, 2))
    # keys and values of kept positions are those of the longer prompt's prefill, whose sums the shorter
    # prompt's own prefill may order differently: the same rollback without sharing is the reference
    t = session(pair)
    t.prefill([2], [prompt])
    t.rollback(2, new_len)
    same(rounds(t, 2, 2), got2)
    s.close()
    t.close()


def test_rollback_clears_its_copy_and_nothing_shared():
    cfg, pair = models("fp32")
    prompt = uniform_prompts(cfg.seed + 4, [53], cfg.target.vocab)[0]
    s = session(pair)
    s.prefill([1], [prompt])
    s.fork(1, [2])
    torch.cuda.synchronize()
    shape, n_pages = cfg.target, s.cache.num_pages_target
    view = lambda: s.kv_target.view(torch.float32).view(shape.n_layers, 2, n_pages, shape.n_kv_heads, 16, shape.head_dim)  # noqa: E731
    before, pages = view().clone(), s.seq_info(1)["pages_target"]
    s.rollback(2, 21)
    torch.cuda.synchronize()
    now, copy = view(), s.seq_info(2)["pages_target"][1]
    assert torch.equal(now[:, :, pages], before[:, :, pages])
    k, v = now[:, 0, copy], now[:, 1, copy].flatten(-2).view(shape.n_layers, shape.n_kv_heads, shape.head_dim, 16)
    kb, vb = before[:, 0, pages[1]], before[:, 1, pages[1]].flatten(-2).view(shape.n_layers, shape.n_kv_heads, shape.head_dim, 16)
    assert torch.equal(k[:, :, :5], kb[:, :, :5]) and torch.equal(v[..., :5], vb[..., :5])
    assert not k[:, :, 5:].any() and not v[..., 5:].any()
    s.close()


def status_of(f):
    from paper_2607_20507_amd import binding as B
    with pytest.raises(B.SpecError) as e:
        f()
    return e.value.status


def test_page_shortage_changes_nothing():
    from paper_2607_20507_amd import binding as B
    cfg, pair = models("fp32")
    prompts = uniform_prompts(cfg.seed + 5, [41, 49], cfg.target.vocab)
    s = session(pair, pages=5)
    s.prefill([1], prompts[:1])  # 40 positions: 3 pages
    assert status_of(lambda: s.fork(1, [2, 3, 4])) == B.SPEC_E_NOPAGES
    s.fork(1, [2, 3])  # a page each: none left
    before = [s.seq_info(i) for i in (1, 2, 3)]
    assert status_of(lambda: s.fork(1, [4])) == B.SPEC_E_NOPAGES
    assert [s.seq_info(i) for i in (1, 2, 3)] == before
    s.rollback(2, 29)  # its own third page makes room for the copy of the shared second
    s.rollback(3, 29)
    s.rollback(1, 29)  # the second page is its own by now: no copy, a page is free
    s.fork(1, [4])
    assert status_of(lambda: s.fork(1, [5])) == B.SPEC_E_NOPAGES
    s.close()
    s = session(pair, pages=3)
    s.prefill([1], prompts[1:])  # 48 positions: 3 full pages
    s.fork(1, [2])
    before = [s.seq_info(i) for i in (1, 2)]
    assert status_of(lambda: s.rollback(2, 20)) == B.SPEC_E_NOPAGES
    assert [s.seq_info(i) for i in (1, 2)] == before
    s.release(1)
    s.rollback(2, 20)
    t = session(pair)
    t.prefill([2], prompts[1:])
    t.rollback(2, 20)
    same(rounds(s, 2, 1), rounds(t, 2, 1))
    s.close()
    t.close()


def test_refusals():
    from paper_2607_20507_amd import binding as B
    cfg, pair = models("fp32")
    prompt = uniform_prompts(cfg.seed + 6, [20], cfg.target.vocab)[0]
    s = session(pair, seqs=3)
    s.prefill([1], [prompt])
    status = status_of
    assert status(lambda: s.fork(9, [2])) == B.SPEC_E_INVALID       # unknown
    assert status(lambda: s.fork(1, [1])) == B.SPEC_E_INVALID       # live
    assert status(lambda: s.fork(1, [2, 2])) == B.SPEC_E_INVALID    # twice
    assert status(lambda: s.fork(1, [2, 3, 4])) == B.SPEC_E_INVALID  # more than max_seqs
    s.fork(1, [])
    s.draft_step([1], [1.0], 1)
    assert status(lambda: s.fork(1, [2])) == B.SPEC_E_STATE          # holds drafts
    na, _ = s.verify([1], [1.0], 1)
    assert status(lambda: s.fork(1, [2])) == B.SPEC_E_STATE          # uncommitted
    s.commit([1], na)
    s.fork(1, [2])
    s.target_forward([2])
    assert status(lambda: s.fork(2, [3])) == B.SPEC_E_STATE          # rows beyond its length
    s.close()


@pytest.mark.parametrize("which", ["fp32", "bf16"])
def test_compaction(which):
    cfg, pair = models(which)
    prompts = uniform_prompts(cfg.seed + 7, [90, 37, 120, 64, 18], cfg.target.vocab)
    s = session(pair)
    s.prefill([1, 2, 3, 4, 5], prompts)
    s.fork(3, [6])
    s.release(1)
    s.release(4)
    s.rollback(3, 100)
    say("compact", which)
    assert s.compact() == s.compact()  # the second moves nothing
    t, d = s.compact()
    held = {side: {p for i in (2, 3, 5, 6) for p in s.seq_info(i)[side]} for side in ("pages_target", "pages_draft")}
    assert held["pages_target"] == set(range(t)) and held["pages_draft"] == set(range(d))
    assert s.seq_info(6)["pages_target"][:6] == s.seq_info(3)["pages_target"][:6]  # still shared
    # contents moved with the names: the pools beyond the pages in use may be overwritten
    torch.cuda.synchronize()
    for kv, shape, n, used in ((s.kv_target, cfg.target, s.cache.num_pages_target, t), (s.kv_draft, cfg.draft, s.cache.num_pages_draft, d)):
        per = shape.n_kv_heads * 16 * shape.head_dim * (4 if shape.dtype == "f32" else 2)
        kv.view(-1, n, per)[:, used:] = 0x7F
    ref = session(pair)
    ref.prefill([1, 2, 3, 4, 5], prompts)
    ref.fork(3, [6])
    ref.rollback(3, 100)
    for sid in (2, 5, 6, 3):
        same(rounds(s, sid, 2), rounds(ref, sid, 2))
    s.prefill([7], [prompts[0]])
    same(rounds(s, 7, 1), alone(pair, prompts[0], 7, 1))
    s.close()
    ref.close()


def test_compaction_between_verify_and_commit():
    cfg, pair = models("bf16")
    prompts = uniform_prompts(cfg.seed + 8, [70, 45], cfg.target.vocab)
    got = []
    for compact in (False, True):
        s = session(pair)
        s.prefill([1, 2], prompts)
        s.draft_loop([2], [0.8], 3, [4])
        s.release(1)
        if compact:
            s.compact()
        na, tok = s.verify([2], [0.8], 3)
        if compact:
            s.compact()
        s.commit([2], na)
        got.append([(int(na[0]), tok[0].tolist(), s.last_logits().cpu().numpy())] + rounds(s, 2, 2, seed=9))
        s.close()
    same(*got)


def test_many_pages_at_once():
    """More moves than travel in a kernel's arguments."""
    cfg, pair = models("fp32")
    from paper_2607_20507_amd.session import SpecSession
    s = SpecSession(pair[0], None, max_seqs=3, k_max=1, max_pages_per_seq=520, max_rows=512, num_pages_target=1100)
    prompts = uniform_prompts(cfg.seed + 9, [8000, 7000], cfg.target.vocab)
    s.prefill([1], prompts[:1])
    s.prefill([2], prompts[1:])
    s.release(1)
    used, draft = s.compact()
    assert used == 438 and draft == 0 and set(s.seq_info(2)["pages_target"]) == set(range(438))
    t = SpecSession(pair[0], None, max_seqs=3, k_max=1, max_pages_per_seq=520, max_rows=512, num_pages_target=1100)
    t.prefill([2], prompts[1:])
    assert np.array_equal(s.decode([2], [0.8], 4, 5), t.decode([2], [0.8], 4, 5))
    s.close()
    t.close()


def test_a_beam_step_with_scores():
    """Alternatives of the last row, a fork for each, their scores: the operators together, against a
    context in which every candidate was prefilled with its token."""
    cfg, pair = models("fp32")
    from oracle.decoder import Decoder
    prompt = uniform_prompts(cfg.seed + 10, [33], cfg.target.vocab)[0]
    s = session(pair, draft=False)
    s.prefill([1], [prompt])
    s.target_forward([1])
    _, entropy, ids, top = s.token_logprobs(n_top=3)
    ref = Decoder(cfg.target, model_weights(cfg.target, cfg.seed))
    z = torch.from_numpy(np.asarray(ref_logits(ref, prompt)))
    want = torch.log_softmax(z.double(), -1)
    assert ids[0].tolist() == torch.topk(want, 3)[1].tolist()
    assert torch.allclose(top[0].double().cpu(), torch.topk(want, 3)[0], atol=2e-3)
    assert abs(float(entropy[0]) - float(-(want.exp() * want).sum())) < 2e-3
    s.verify([1], [0.0], 1)
    s.rollback(1, len(prompt) - 1)
    s.fork(1, [2, 3, 4])
    for sid, tok in zip((2, 3, 4), ids[0].tolist()):
        s.set_drafts(sid, [tok], torch.zeros(1, cfg.target.vocab, device=s.kv_target.device))
    s.target_forward([2, 3, 4])  # two rows each: the pending token's, the candidate's
    lp, _, ids2, top2 = s.token_logprobs(tokens=[t for tok in ids[0].tolist() for t in (tok, 0)], n_top=2)
    assert torch.allclose(lp[0::2], top[0], atol=1e-4)
    for j, tok in enumerate(ids[0].tolist()):
        w = torch.log_softmax(torch.from_numpy(np.asarray(ref_logits(ref, list(prompt) + [tok]))).double(), -1)
        assert ids2[2 * j + 1].tolist() == torch.topk(w, 2)[1].tolist()
        assert torch.allclose(top2[2 * j + 1].double().cpu(), torch.topk(w, 2)[0], atol=2e-3)
    s.close()


def ref_logits(decoder, tokens):
    return decoder.full_logits(np.asarray(tokens))[-1]
