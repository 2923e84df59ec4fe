"""Attention over a latent cache against its definition in 64 bits."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_20507_amd import binding as B  # noqa: E402
from tests import latent_ref as L  # noqa: E402
from tests.gpu_util import device, say  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
BIG, SMALL = dict(nope=128, rope=64, rank=512, v=128), dict(nope=64, rope=32, rank=256, v=64)


def check(c, ws=None):
    got = c.run(B, ws)
    ref = c.ref()
    assert torch.isfinite(got).all()
    assert (c.out[len(c.q):] == 7).all()  # nothing behind the last row
    err = L.row_error(got, ref)
    say("error", err)
    assert err <= L.TOL[c.dtype], err


# rows, first positions, heads: one token to long contexts, odd head counts (tiles that end inside a row's heads),
# sequences without rows, contexts that end inside a page, at one and one past
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sizes", [BIG, SMALL], ids=["512", "256"])
@pytest.mark.parametrize("rows, pos0, H", [
    ([1], [0], 1), ([1], [0], 32), ([1], [15], 16), ([1], [16], 5), ([2], [30], 16), ([1], [1000], 16), ([1], [1000], 32),
    ([1], [777], 40), ([1], [2500], 128), ([6], [2047], 32), ([5], [128], 4), ([1, 1, 1], [5, 300, 31], 16),
    ([4, 0, 6, 8], [100, 9, 515, 64], 11), ([0, 3], [0, 0], 7), ([17], [0], 12), ([33, 2], [0, 95], 32), ([70], [50], 3)])
def test_attention(dtype, sizes, rows, pos0, H):
    device()
    say("latent attention", dtype, sizes, rows, pos0, H)
    check(L.Case(dtype, rows, pos0, H, seed=sum(rows) + H, **sizes))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("nope, rope, rank, v", [(64, 64, 512, 128), (128, 32, 512, 64), (64, 32, 512, 64), (128, 64, 256, 128),
                                                 (128, 32, 256, 64), (64, 64, 256, 128)])
def test_sizes(dtype, nope, rope, rank, v):
    device()
    say("sizes", dtype, nope, rope, rank, v)
    for rows, pos0, H in [([1], [400], 9), ([5, 2], [70, 333], 20), ([290, 3, 517], [111, 80, 0], 3)]:
        check(L.Case(dtype, rows, pos0, H, nope, rope, rank, v, seed=5))


# many sequences of few rows: products of 47 rows and more at a time, with last blocks of one row, of 16 and of others
@pytest.mark.parametrize("sizes", [BIG, SMALL, dict(nope=64, rope=64, rank=512, v=64)], ids=["512", "256", "mixed"])
@pytest.mark.parametrize("seqs, most, H", [(47, 1, 8), (48, 1, 3), (49, 1, 16), (20, 8, 5), (70, 6, 16), (40, 23, 1), (130, 8, 1)])
def test_many_sequences(sizes, seqs, most, H):
    device()
    say("many", sizes, seqs, most, H)
    rng = np.random.default_rng(seqs)
    rows = rng.integers(most if most == 1 else 0, most + 1, seqs).tolist()
    check(L.Case(BF, rows, rng.integers(0, 200, seqs).tolist(), H, seed=seqs, **sizes))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_context(dtype):
    device()
    for rows, H in [(1, 32), (3, 16)]:
        say("long", dtype, rows, H)
        check(L.Case(dtype, [rows], [30001], H, seed=6))


# long runs of rows, alone and beside sequences of a few
@pytest.mark.parametrize("rows, pos0, H", [([300], [0], 32), ([257, 100], [513, 40], 16), ([1024], [100], 5), ([90, 1], [3000, 200], 32),
                                           ([3, 600, 0, 1, 256, 5], [70, 33, 4, 1000, 0, 31], 7), ([2000], [5], 2)])
@pytest.mark.parametrize("dtype, sizes", [(BF, BIG), (BF, SMALL), (F32, SMALL)], ids=["bf16-512", "bf16-256", "f32-256"])
def test_prompts(dtype, sizes, rows, pos0, H):
    device()
    say("prompt", dtype, sizes, rows, pos0, H)
    check(L.Case(dtype, rows, pos0, H, seed=8, **sizes))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows, H", [(6, 16), (200, 4), (400, 3)])
def test_one_key_far_above_the_others(dtype, rows, H):
    """Scores spread over hundreds: a row's weight is one key's, found late in its context."""
    device()
    say("peak", dtype, rows, H)
    c = L.Case(dtype, [rows], [700], H, seed=9)
    c.q *= 64
    flat = c.pages.view(-1, 576)
    flat[c.slots(0)[650]] *= 3
    got, ref = c.run(B), c.ref()
    # scores' deviation is 64 to 200 here: their roundings (64 to 200 times 0.0017 in bf16) move weight between the leading keys,
    # so a row is compared where one key leads by e^24, which no such rounding outweighs
    sc = []
    held = flat[c.slots(0)].double()
    for h in range(H):
        k = torch.cat([held[:, :512] @ c.w_k[h].double().t().contiguous(), held[:, 512:]], 1)
        s = c.q[:, h].double() @ k.t().contiguous() * c.scale
        s.masked_fill_(torch.arange(len(held), device="cuda") > 700 + torch.arange(rows, device="cuda")[:, None], -math.inf)
        top = s.topk(2, 1)[0]
        sc.append(top[:, 0] - top[:, 1] > 24)
    lead = torch.stack(sc, 1)
    assert int(lead.sum()) > 10 and torch.isfinite(got).all()
    assert L.row_error(got[lead], ref[lead]) <= L.TOL[dtype]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("power", [7, 14, 22])
@pytest.mark.parametrize("rows, pos0", [(3, 500), (3, 5000), (200, 3), (40, 3000)])
def test_large_logits_keep_small_differences(dtype, power, rows, pos0):
    """Logits of 2^power + 0 .. 3, whose products and sums 24 bits hold exactly: e^0 .. e^-3 once the maximum is taken away."""
    device()
    say("large", dtype, power, rows, pos0)
    c = L.Case(dtype, [rows], [pos0], 4, seed=19, **SMALL)
    flat = c.pages.view(-1, 288)
    n = rows + pos0
    g = torch.Generator(device="cuda")
    g.manual_seed(20)
    level = torch.randint(0, 4, (n,), generator=g, device="cuda")
    flat[c.slots(0), 256:] = 0
    flat[c.slots(0), 256] = 1
    flat[c.slots(0), 257] = level.to(dtype)
    c.q.zero_()
    c.q[:, :, 64] = 2.0 ** power
    c.q[:, :, 65] = 1
    c.scale = 1.0
    got, ref = c.run(B), c.ref()
    assert torch.isfinite(got).all() and L.row_error(got, ref) <= L.TOL[dtype]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows, pos0", [(3, 500), (200, 3)])
def test_a_scale_that_makes_logits_huge(dtype, rows, pos0):
    """Logits to 2^30 and beyond: a row is its best key's value, at differences of thousands and more."""
    device()
    say("huge", dtype, rows, pos0)
    c = L.Case(dtype, [rows], [pos0], 4, seed=21, **SMALL)
    c.scale = 1e9
    got, ref = c.run(B), c.ref()
    assert torch.isfinite(got).all()
    flat, r = c.pages.view(-1, 288), torch.arange(rows, device="cuda")
    held = flat[c.slots(0)].double()
    for h in range(4):
        k = torch.cat([held[:, :256] @ c.w_k[h].double().t().contiguous(), held[:, 256:]], 1)
        s = c.q[:, h].double() @ k.t().contiguous()
        s.masked_fill_(torch.arange(len(held), device="cuda") > pos0 + r[:, None], -math.inf)
        # one rounding to bf16 of queries or keys moves a score by 0.0017 sqrt(64) in the root mean square, two scores' difference
        # by 0.02: 0.3 is 15 times that
        top = s.topk(min(2, s.shape[1]), 1)[0]
        lead = top[:, 0] - top[:, -1] > 0.3
        assert int(lead.sum()) >= min(rows, 50) // 3
        assert L.row_error(got[lead, h], ref[lead, h]) <= L.TOL[dtype]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H", [4, 16, 32])
@pytest.mark.parametrize("where, value", [("latent", math.nan), ("latent", -math.inf), ("key", math.nan), ("key", math.inf)])
@pytest.mark.parametrize("rows, bad", [(6, 3), (300, 3), (300, 150), (300, 290)])
def test_entries_that_are_not_finite_reach_the_rows_that_see_them(dtype, H, where, value, rows, bad):
    device()
    say("not finite", dtype, H, where, value, rows, bad)
    c = L.Case(dtype, [rows, 2], [200, 31], H, seed=10, **SMALL)
    flat = c.pages.view(-1, 288)
    flat[c.slots(0)[200 + bad], 17 if where == "latent" else 260] = value  # the key of row `bad`
    got, ref = c.run(B), c.ref()
    fine = torch.isfinite(ref).all(-1)
    assert fine[:bad].all() and fine[rows:].all()
    assert torch.isfinite(got[fine]).all() and L.row_error(got[fine], ref[fine]) <= L.TOL[dtype]
    assert not torch.isfinite(got[~fine]).all(-1).any()
    if where == "latent" or math.isnan(value):
        assert not fine[bad:rows].any()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_shared_key_of_minus_infinity_is_not_attended(dtype):
    """Its scores are -inf for queries of the same sign there and +inf for the others, whose rows are NaN."""
    device()
    say("masked key", dtype)
    c = L.Case(dtype, [4], [100], 8, seed=11, **SMALL)
    c.q[:, :, 64 + 5] = c.q[:, :, 64 + 5].abs() + 0.5
    c.q[2, 3, 64 + 5] *= -1
    c.pages.view(-1, 288)[c.slots(0)[40], 256 + 5] = -math.inf
    got, ref = c.run(B), c.ref()
    fine = torch.isfinite(ref).all(-1)
    assert int((~fine).sum()) == 1 and not fine[2, 3]
    assert L.row_error(got[fine], ref[fine]) <= L.TOL[dtype] and torch.isnan(got[~fine]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_batch_composition_and_repeats(dtype):
    """The same bits from call to call, with a workspace that held another call's values."""
    device()
    say("repeats", dtype)
    c = L.Case(dtype, [6, 1, 400, 4], [1500, 20, 700, 333], 16, seed=12)
    ws = c.workspace(B)
    first = c.run(B, ws).clone()
    for _ in range(3):
        c.out.zero_()
        assert torch.equal(c.run(B, ws), first)


def test_page_ids_beyond_32_bit_offsets():
    """A pool of more than 2^32 bytes, its last pages in use."""
    device()
    say("large pool")
    c = L.Case(BF, [2, 300], [100, 0], 16, seed=13)
    P = (1 << 32) // (16 * 576 * 2) + 40
    pages = torch.zeros(P, 16, 576, dtype=BF, device="cuda")
    used = int(c.table.max()) + 1
    pages[P - used:] = c.pages[:used]
    ref = c.ref()
    c.table, c.pages, c.P = np.where(c.table >= 0, c.table + P - used, -1).astype(np.int32), pages, P
    assert L.row_error(c.run(B), ref) <= L.TOL[BF]


def test_expanded_pages_up_to_their_limit():
    """Keys and values of 60500 tokens of 128 heads, 3.96 GB beyond 32-bit offsets; a second prompt's would pass 4 GiB, and it is
    attended to in the cache itself."""
    device()
    say("4 GiB")
    H, rows, pos0 = 128, [5500, 5200], [55000, 0]
    c = L.Case(BF, rows, pos0, H, seed=23)
    one = B.spec_op_attention_latent_workspace_bytes(B.SPEC_BF16, rows[:1], pos0[:1], c.table.shape[1], H, 128, 64, 512, 128)
    both = B.spec_op_attention_latent_workspace_bytes(*c.args(B), c.table.shape[1], H, 128, 64, 512, 128)
    say("workspace", one, both)
    assert one > 60500 * H * 512 and both - one >= 2 * 5200 * H * 1024  # the second: queries and sums in the latents' space
    got = c.run(B)
    flat, first = c.pages.view(-1, 576), 0
    for i in range(2):
        held = flat[c.slots(i)]
        for r in (0, 127, 2700, rows[i] - 2):  # two rows from each
            n = pos0[i] + r + 2
            ref = L.attend(c.q[first + r:first + r + 2], held[:n], pos0[i] + r, c.w_k, c.w_v, c.scale, 512)
            err = L.row_error(got[first + r:first + r + 2], ref)
            say("error", i, r, err)
            assert err <= L.TOL[BF]
        first += rows[i]
    assert torch.isfinite(got).all() and (c.out[len(c.q):] == 7).all()


def test_two_calls_at_once():
    """Two streams, each with a workspace of its own, a verify beside a prompt, again and again."""
    device()
    say("two calls")
    cases = [L.Case(BF, [6, 5], [2047, 300], 32, seed=24), L.Case(BF, [700], [100], 8, seed=25)]
    spaces, refs = [c.workspace(B) for c in cases], [c.run(B).clone() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        for c, ws, st in zip(cases, spaces, streams):
            c.out.fill_(7)
        torch.cuda.synchronize()
        for _ in range(4):
            for c, ws, st in zip(cases, spaces, streams):
                c.run(B, ws, st)
        torch.cuda.synchronize()
        for c, ref in zip(cases, refs):
            assert torch.equal(c.out[:len(c.q)].view_as(ref), ref)
    for c, ref in zip(cases, refs):
        assert L.row_error(ref, c.ref()) <= L.TOL[BF]


@pytest.mark.parametrize("case", [([6], [2047]), ([2, 300], [40, 100])], ids=["verify", "mixed"])
def test_another_stream_and_a_captured_call(case):
    device()
    say("stream and graph")
    rows, pos0 = case
    n = sum(rows)
    c = L.Case(BF, rows, pos0, 32, seed=14)
    want = c.run(B).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    ws = c.workspace(B)
    side.wait_stream(torch.cuda.current_stream())
    c.run(B, ws, side)
    side.synchronize()
    assert torch.equal(c.out[:n].view(n, 32, 128), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(B, ws)
    other = L.Case(BF, [3], [50], 7, seed=15)
    for i in range(4):  # new inputs in the captured buffers, other work between the replays
        g = torch.Generator(device="cuda")
        g.manual_seed(i)
        c.q.copy_(torch.randn(c.q.shape, generator=g, device="cuda"))
        c.out.zero_()
        graph.replay()
        got = c.out[:n].clone()
        other.run(B)
        torch.cuda.synchronize()
        c.out.zero_()
        c.run(B)
        assert torch.equal(got, c.out[:n])


def test_a_captured_call_with_large_tables_is_refused():
    device()
    say("capture refused")
    c = L.Case(BF, [1] * 8, [2000] * 8, 4, seed=16, **SMALL)
    ws = c.workspace(B)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(B.SpecError) as e:
        with torch.cuda.graph(graph):
            c.run(B, ws)
    assert e.value.status == B.SPEC_E_UNSUPPORTED
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_and_attention_as_a_model_calls_them(dtype):
    """A prompt in two chunks, a verify, a rollback, a decoded token: each layer call appends, then attends; a fork's pages are
    copied and go on by themselves."""
    device()
    H, nope, rope, rank, v = 6, 64, 32, 256, 64
    theta, eps = 1e4, 1e-5
    dt = B.SPEC_F32 if dtype is F32 else B.SPEC_BF16
    g = torch.Generator(device="cuda")
    g.manual_seed(17)
    P = 34
    pool = torch.full((1, P, 16, rank + rope), math.nan, dtype=dtype, device="cuda")
    w = (torch.randn(H, nope + v, rank, generator=g, device="cuda") / 16).to(dtype)
    norm_w = (1 + 0.1 * torch.randn(rank, generator=g, device="cuda")).to(dtype)
    table = np.random.default_rng(3).permutation(P)[:28].astype(np.int32)
    fork = np.setdiff1d(np.arange(P), table).astype(np.int32)
    held = torch.empty(0, rank + rope, dtype=torch.float64, device="cuda")
    scale = 1 / math.sqrt(nope + rope)

    def step(table, held, rows):
        n = len(held)
        q = torch.randn(rows, H, nope + rope, generator=g, device="cuda")
        kv = torch.randn(rows, rank + rope, generator=g, device="cuda")
        at = n + np.arange(rows)
        pos = torch.from_numpy(at.astype(np.int32)).to("cuda")
        slot = torch.from_numpy((table[at // 16] * 16 + at % 16).astype(np.int32)).to("cuda")
        q_out, out = torch.empty(rows, H, nope + rope, dtype=dtype, device="cuda"), torch.empty(rows, H * v, dtype=dtype, device="cuda")
        B.spec_op_rope_latent(dt, rows, H, nope, rope, rank, theta, eps, q, kv, norm_w, pos, slot, P, q_out, pool)
        nb = B.spec_op_attention_latent_workspace_bytes(dt, [rows], [n], len(table), H, nope, rope, rank, v)
        ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
        B.spec_op_attention_latent(dt, [rows], [n], table[None], P, H, nope, rope, rank, v, scale, q_out, pool, w[:, :nope],
                                   w[:, nope:], out, ws)
        rq, entry = L.append(q, kv, norm_w, pos, H, nope, rope, rank, theta, eps)
        held = torch.cat([held, entry.to(dtype).double()])
        ref = L.attend(rq.to(dtype), held, n, w[:, :nope], w[:, nope:], scale, rank)
        err = L.row_error(out.view(rows, H, v), ref)
        say("step", dtype, n, rows, err)
        # a value that fp32 and fp64 round to different bf16 neighbours is one more rounding of a few inputs
        assert err <= L.TOL[dtype]
        return held

    held = step(table, held, 277)
    held = step(table, held, 77)
    held = step(table, held, 6)
    held = held[:356]  # two of six drafts kept
    held = step(table, held, 1)
    # a fork shares the full pages and copies the last
    last = len(held) // 16
    mine = np.concatenate([table[:last], fork[:4]]).astype(np.int32)
    ws = torch.empty(max(256, B.spec_op_kv_copy_pages_workspace_bytes(1)), dtype=torch.uint8, device="cuda")
    B.spec_op_kv_copy_pages(pool, [table[last]], [mine[last]], ws)
    other = step(mine, held, 3)
    held = step(table, held, 3)
    step(mine, other, 1)
    step(table, held, 1)
