"""Attention over the 4-bit cache on a GPU against float64, with an error bound of
its own for each row, head and dim, which an output of zeros, of the wrong sign
or of another head does not meet."""

import functools

import numpy as np
import pytest

import kv4_ref as ref
from gpu_util import device, say
from test_gpu_kv4 import BF16, F32, HALF_STEP, TYPES, attend, to

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def rel_bound(dtype, hd, n, big):
    """Relative error of a row's probabilities and sums.

    Scores: products of bf16 numbers are exact in fp32 (q in three parts for fp32: three times as many), each of
    their additions is off by at most 2^-24 of sum |q k|; the scale (its own 3 roundings), the product with it and
    the difference to the maximum add 5 more: (c hd + 5) 2^-24 sum |q k| / sqrt(hd) absolutely, which is a relative
    error of exp.  It enters the numerator and the denominator.  The exponent's own rounding is below 150 2^-24 (p
    below 2^-150 is 0), exp2 has 2^-22, as has every factor that moves sums to a new maximum or joins waves and
    parts: with n keys fewer than n / 32 + 80 of those.  n additions (3 n for three parts) of 2^-24 each.  The
    probabilities that meet V are rounded to bf16, or to 24 bits."""
    c = 3 if dtype == F32 else 1
    score = (c * hd + 5) * 2.0 ** -24 * big
    return 2 * score + (150 + 4 * (n / 32 + 80) + c * n) * 2.0 ** -24 + HALF_STEP[dtype]


def bound(dtype, hd, n, want, mag, big):
    rel = rel_bound(dtype, hd, n, big)
    assert np.max(rel) < 0.03
    # (numerator and denominator off by rel each, products of errors below 4%; the output's rounding)
    return 1.04 * (rel * (mag + np.abs(want)) + HALF_STEP[dtype] * np.abs(want))


def vectors(rng, *shape):
    x = rng.standard_normal(shape)
    x[..., 3::17] *= 8  # a few dims much larger, as keys have them
    if shape[0] > 4:
        x[1, 0, :32] = 0
        x[2, 0, 32:64] *= 1e-20
    return x.astype(np.float32).astype(np.float64)


@functools.lru_cache(maxsize=None)
def places(place, hd):
    """[16, hd] bytes, nibbles and scale bytes of a block."""
    at = np.array([[place(t, d, hd) for d in range(hd)] for t in range(16)])
    return at[..., 0], at[..., 1], at[..., 2]


def store(pool, slot, x, place):
    """Vectors x [n, Hkv, hd] into the slots of pages whose codes are 0, and the values that they hold."""
    n, hkv, hd = x.shape
    b = x.reshape(n, hkv, -1, 32)
    top = np.abs(b).max(-1)
    e = np.maximum(np.frexp(top)[1] - 3, -126)
    e += 6.0 * 2.0 ** e < top
    code = np.abs(np.abs(b)[..., None] * 2.0 ** -e[..., None, None].astype(float) - ref.LEVELS).argmin(-1) + 8 * np.signbit(b)
    byte, nib, sb = (a[slot % 16] for a in places(place, hd))
    page = slot[:, None] // 16
    flat = code.reshape(n, hkv, hd)
    for h in range(hkv):
        for half in (0, 1):  # a byte holds one value of each nibble
            r, d = np.nonzero(nib == half)
            pool[page[r, 0], h, byte[r, d]] |= (flat[r, h, d] << (4 * half)).astype(np.uint8)
        pool[page, h, sb] = np.repeat(e[:, h] + 127, 32, -1)
    return (ref.SIGNED[code] * 2.0 ** e[..., None]).reshape(n, hkv, hd)


def pages(rng, lens, hkv, hd, dev, k_of, v_of):
    """Pages, page table and fp64 values of sequences with the keys k_of(n) and values v_of(n); the rest is NaN."""
    need = [(n + 15) // 16 for n in lens]
    P = sum(need) + 3
    perm = rng.permutation(P)
    table = np.full((len(lens), max(max(need), 1)), -1, np.int32)
    pools = [np.full((P, hkv, ref.block_bytes(hd)), 0xFF, np.uint8) for _ in range(2)]
    values = []
    for i, (n, o) in enumerate(zip(lens, np.cumsum(need) - need)):
        table[i, :need[i]] = perm[o:o + need[i]]
        slot = table[i][np.arange(n) // 16] * 16 + np.arange(n) % 16
        kv = []
        for pool, place, of in zip(pools, (ref.k_place, ref.v_place), (k_of, v_of)):
            x = of(n)
            pool[table[i, :need[i]], :, :8 * hd] = 0
            kv.append(store(pool, slot, x, place) if n else x)
        values.append(kv)
    return table, pools, values


def fits(got, want, tol):
    with np.errstate(invalid="ignore"):
        return bool(np.all(np.abs(got - want) <= tol))


def check(dtype, rows, pos0, hq, hkv, hd, only=None, shared=False):
    dev = device()
    say("4-bit attention", dtype, hq, hkv, hd, rows[:8], pos0[:8])
    rng = np.random.default_rng([hq, hd, len(rows), sum(rows), pos0[0]])
    lens = [r + p if r else 0 for r, p in zip(rows, pos0)]
    of = lambda n: vectors(rng, n, hkv, hd)  # noqa: E731
    if shared:  # every sequence over the same keys
        table, (kp, vp), ((k, v),) = pages(rng, [max(lens)], hkv, hd, dev, of, of)
        table, values = np.repeat(table, len(lens), 0), [(k[:n], v[:n]) for n in lens]
    else:
        table, (kp, vp), values = pages(rng, lens, hkv, hd, dev, of, of)
    q = to(dev, rng.standard_normal((sum(rows), hq, hd)) * 1.5, TYPES[dtype])
    got = attend(dtype, rows, pos0, table, len(kp), hq, hkv, hd, q, to(dev, kp, torch.uint8), to(dev, vp, torch.uint8), dev)
    got, q64 = got.double().cpu().numpy().reshape(-1, hq, hd), q.double().cpu().numpy()
    r0 = 0
    for i, (r, p) in enumerate(zip(rows, pos0)):
        if r and (only is None or i in only):
            want, mag, big = ref.attention_rows(q64[r0:r0 + r], *values[i], p)
            tol = bound(dtype, hd, r + p, want, mag, big)
            g = got[r0:r0 + r]
            assert fits(g, want, tol), (i, float(np.max(np.abs(g - want) / tol)))
            # the bound tells right from wrong: most elements by far
            assert np.mean(np.abs(want[want != 0]) > 4 * tol[want != 0]) > 0.7 and np.mean(want != 0) > 0.3
            for wrong in (0 * g, -g, np.roll(g, 1, 2)) + ((np.roll(g, 1, 1),) if hq > 1 and (r + p > 1 or hq == hkv > 1) else ()):
                assert not fits(wrong, want, tol)
        r0 += r


HEADS = [(F32, 4, 4, 64), (F32, 8, 2, 128), (F32, 32, 1, 64), (BF16, 16, 16, 64), (BF16, 32, 8, 128), (BF16, 32, 8, 64),
         (BF16, 7, 1, 64), (BF16, 6, 2, 128), (BF16, 16, 1, 128), (BF16, 64, 1, 64)]


@pytest.mark.parametrize("dtype, hq, hkv, hd", HEADS)
@pytest.mark.parametrize("rows, pos0", [
    ([1], [0]), ([1], [15]), ([2], [31]), ([6], [500]), ([3, 0, 8, 1], [0, 40, 29, 128]), ([17, 5], [3, 640]), ([0, 1], [9, 2])])
def test_rows(dtype, hq, hkv, hd, rows, pos0):
    check(dtype, rows, pos0, hq, hkv, hd)


@pytest.mark.parametrize("dtype, hq, hkv, hd", [(F32, 4, 4, 64), (BF16, 8, 2, 128), (BF16, 32, 8, 64), (BF16, 64, 1, 64)])
@pytest.mark.parametrize("rows, pos0", [([1], [1290]), ([1], [9000]), ([6], [5000]), ([2, 1], [700, 4100])])
def test_split_contexts(dtype, hq, hkv, hd, rows, pos0):
    check(dtype, rows, pos0, hq, hkv, hd)


def test_many_parts():
    check(BF16, [1], [40000], 8, 2, 128)
    check(F32, [1], [20000], 4, 2, 64)


@pytest.mark.parametrize("dtype, hq, hkv, hd", [(BF16, 32, 8, 128), (BF16, 8, 8, 64), (F32, 8, 4, 64)])
def test_batches(dtype, hq, hkv, hd):
    """More work items than CUs, of uneven lengths."""
    n = 40
    pos0 = [37 * i % 1500 for i in range(n)]
    check(dtype, [1 + i % 5 for i in range(n)], pos0, hq, hkv, hd, only=(0, 7, 13, 27, 39))


def test_items_of_more_keys_than_staged_page_ids():
    """32 sequences over one long prefix: whole items of 20000 keys, 1250 pages."""
    check(BF16, [2] * 32, [20000 - 37 * i for i in range(32)], 32, 8, 64, only=(0, 31), shared=True)


@pytest.mark.parametrize("dtype, hq, hkv, hd", [(F32, 4, 4, 64), (BF16, 8, 2, 128), (BF16, 4, 2, 64), (BF16, 7, 1, 64), (BF16, 64, 1, 128)])
@pytest.mark.parametrize("rows, pos0", [([63], [5]), ([64], [0]), ([70, 130], [0, 33]), ([300], [100]), ([64, 0, 65], [400, 3, 0]), ([64, 3], [200, 90])])
def test_prompts(dtype, hq, hkv, hd, rows, pos0):
    check(dtype, rows, pos0, hq, hkv, hd)


def test_a_prompt_chunk_behind_many_keys():
    check(BF16, [64], [16400], 8, 2, 64)  # beyond the prompt form's 16384 keys
    check(BF16, [64], [9000], 8, 2, 128)


# ---------------------------------------------------------------------------
# Scores of 2^17 to 2^25 in base 2, whose differences are a few units: sums of a few numbers that fp32 holds
# exactly in any order, so that the scores have no error and only their differences count.

def far_keys(rng, n, hkv, hd, unit):
    """Dims 0 .. 2: 1; dim 32: a multiple of `unit`, small for most keys, larger for some of the later ones."""
    k = np.zeros((n, hkv, hd))
    k[..., :3] = 1
    fine = rng.choice([0, 1, 2, 3], (n, hkv))
    late = (np.arange(n)[:, None] > n // 3) & (rng.random((n, hkv)) < 0.02)
    k[..., 32] = np.where(late, rng.choice([6, 8, 12], (n, hkv)), fine) * unit
    return k


def bf16_parts(x):
    """x as a sum of three bf16 numbers."""
    parts = []
    for _ in range(3):
        p = float(torch.tensor(x, dtype=torch.float64).to(torch.bfloat16))
        parts.append(p)
        x -= p
    assert x == 0
    return parts


def border(hd):
    """The score at which the exponent form changes (2^24 in base 2), less a few units of 8."""
    return float(int(2.0 ** 24 / (1.4426950408889634 / hd ** 0.5)) // 8 * 8 - 24)


@pytest.mark.parametrize("dtype, hq, hkv, hd", [(F32, 4, 4, 64), (F32, 8, 2, 128), (BF16, 8, 2, 128), (BF16, 16, 4, 64), (BF16, 64, 1, 64)])
@pytest.mark.parametrize("base", [2.0 ** 20, -2.0 ** 20, 2.0 ** 24, 2.0 ** 26, -2.0 ** 26, "border", 2.0 ** 27, -2.0 ** 27])
@pytest.mark.parametrize("rows, pos0", [(1, 39), (6, 700), (3, 3000), (64, 340), (100, 500)])
def test_scores_far_from_zero(dtype, hq, hkv, hd, base, rows, pos0):
    dev = device()
    base = border(hd) if base == "border" else base
    unit = 16.0 if abs(base) >= 2.0 ** 27 else 8.0
    say("far scores", dtype, hq, hkv, hd, base, rows, pos0)
    rng = np.random.default_rng([hq, hd, rows, pos0])
    table, (kp, vp), ((k, v),) = pages(rng, [rows + pos0], hkv, hd, dev, lambda n: far_keys(rng, n, hkv, hd, unit),
                                       lambda n: rng.standard_normal((n, hkv, hd)).astype(np.float32).astype(np.float64))
    q = np.zeros((rows, hq, hd))
    q[..., :3] = bf16_parts(base)
    q[..., 32] = 1
    got = attend(dtype, [rows], [pos0], table, len(kp), hq, hkv, hd, to(dev, q, TYPES[dtype]), to(dev, kp, torch.uint8),
                 to(dev, vp, torch.uint8), dev).double().cpu().numpy().reshape(rows, hq, hd)
    q[..., :3] = 0  # the same for every key: the softmax is that of the rest
    want, mag, _ = ref.attention_rows(q, k, v, pos0)
    # the scores are exact; their differences, at most 12 units, lose 3 roundings
    tol = bound(dtype, hd, rows + pos0, want, mag, 12 * unit / hd ** 0.5 * 3 / (hd + 5))
    assert fits(got, want, tol), float(np.max(np.abs(got - want) / tol))


# ---------------------------------------------------------------------------
# NaN and infinities

@pytest.mark.parametrize("dtype, hq, hkv, hd", [(F32, 4, 4, 64), (BF16, 64, 1, 64)])
def test_no_part_loses_a_nan(dtype, hq, hkv, hd):
    """A part of a split context (128 keys here) whose scores are all NaN: so is every row."""
    dev = device()
    for n, blocks in ((1290, range(11)), (66 * 128, (0, 5, 63, 64, 65))):
        rng = np.random.default_rng(n)
        of = lambda m: rng.standard_normal((m, hkv, hd))  # noqa: E731
        table, (kp, vp), _ = pages(rng, [n], hkv, hd, dev, of, of)
        kp, vp = to(dev, kp, torch.uint8), to(dev, vp, torch.uint8)
        q = to(dev, rng.standard_normal((1, hq, hd)), TYPES[dtype])
        for b in blocks:
            k = kp.clone()
            k[torch.from_numpy(table[0, 8 * b:8 * b + 8].astype(np.int64)).to(dev)] = 0xFF
            out = attend(dtype, [1], [n - 1], table, len(kp), hq, hkv, hd, q, k, vp, dev)
            assert bool(out.isnan().all()), (n, b)


@pytest.mark.parametrize("dtype, hq, hkv, hd", [(F32, 4, 4, 64), (F32, 8, 2, 128), (BF16, 8, 2, 128), (BF16, 4, 2, 64), (BF16, 64, 1, 64)])
@pytest.mark.parametrize("what", ["nan value", "infinite value", "nan key"])
@pytest.mark.parametrize("rows, pos0, bad", [(8, 40, 43), (8, 40, 47), (17, 20, 31), (5, 1290, 1293), (64, 0, 30), (100, 300, 333), (200, 100, 130), (130, 380, 509)])
def test_keys_that_a_row_does_not_see(dtype, hq, hkv, hd, what, rows, pos0, bad):
    """A NaN or an infinity in a key or value behind a row's position leaves the row as it is."""
    dev = device()
    say("hidden", what, dtype, hq, hkv, hd, rows, pos0, bad)
    rng = np.random.default_rng([rows, pos0, hd])
    n = rows + pos0
    of = lambda m: rng.standard_normal((m, hkv, hd)).astype(np.float32).astype(np.float64)  # noqa: E731
    table, pools, ((k, v),) = pages(rng, [n], hkv, hd, dev, of, of)
    pool, place = (pools[0], ref.k_place) if what == "nan key" else (pools[1], ref.v_place)
    x = np.zeros((1, hkv, hd))
    x[..., 32:64] = np.nan if what[0] == "n" else 1.9 * 2.0 ** 127  # (held as 2^128, an infinity in fp32)
    slot = [table[0, bad // 16] * 16 + bad % 16]
    ref.put(pool, slot, x, place)
    held = ref.get(pool, np.asarray(slot), hd, place)[0]
    (k if what == "nan key" else v)[bad] = np.where(np.abs(held) >= 2.0 ** 128, np.inf, held)
    q = to(dev, rng.standard_normal((rows, hq, hd)), TYPES[dtype])
    got = attend(dtype, [rows], [pos0], table, len(pools[0]), hq, hkv, hd, q, to(dev, pools[0], torch.uint8),
                 to(dev, pools[1], torch.uint8), dev).double().cpu().numpy().reshape(rows, hq, hd)
    want, mag, big = ref.attention_rows(q.double().cpu().numpy(), k, v, pos0)
    assert np.isfinite(want[:bad - pos0]).all() and not np.isfinite(want[bad - pos0:, :, 32:64]).any()
    assert np.array_equal(np.isnan(got), np.isnan(want)), "NaN"
    assert np.array_equal(np.isposinf(got), np.isposinf(want)), "infinities"
    fine = np.isfinite(want)
    big = np.where(np.isfinite(big), big, 0)
    tol = bound(dtype, hd, n, np.where(fine, want, 0), np.where(fine, mag, 0), big)
    assert np.all(np.abs(got[fine] - want[fine]) <= tol[fine])


# ---------------------------------------------------------------------------
# captured calls

@pytest.mark.parametrize("rows, pos0, taken", [([6], [2047], True), ([1], [100], True), ([1], [2600], True), ([3, 2, 4], [50, 900, 20], True),
                                               ([2] * 40, [1500] * 40, False)])
def test_captured_calls(rows, pos0, taken):
    """Tables of up to 3 KB are taken into a graph, whose replays equal eager calls; larger ones are refused."""
    from paper_2607_20507_amd import binding as B
    dev = device()
    hq, hkv, hd, R = 32, 8, 128, sum(rows)
    rng = np.random.default_rng(12)
    of = lambda m: rng.standard_normal((m, hkv, hd))  # noqa: E731
    table, (kp, vp), _ = pages(rng, [r + p for r, p in zip(rows, pos0)], hkv, hd, dev, of, of)
    kp, vp = to(dev, kp, torch.uint8), to(dev, vp, torch.uint8)
    q = torch.empty(R, hq, hd, dtype=torch.bfloat16, device=dev)
    ws = torch.empty(B.spec_op_attention_kv4_workspace_bytes(BF16, rows, pos0, table.shape[1], hq, hkv, hd), dtype=torch.uint8, device=dev)
    out = torch.empty(R, hq * hd, dtype=torch.bfloat16, device=dev)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    call = lambda: B.spec_op_attention_kv4(BF16, rows, pos0, table, kp.shape[0], hq, hkv, hd, q, kp, vp, out, ws, side)  # noqa: E731
    with torch.cuda.graph(graph, stream=side):
        if taken:
            call()
        else:
            out.zero_()
            with pytest.raises(B.SpecError) as e:
                call()
            assert e.value.status == B.SPEC_E_UNSUPPORTED
    if not taken:
        return
    for seed in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator(device=dev).manual_seed(seed), device=dev))
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, attend(BF16, rows, pos0, table, kp.shape[0], hq, hkv, hd, q, kp, vp, dev)), seed
