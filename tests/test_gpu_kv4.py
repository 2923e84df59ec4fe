"""The 4-bit cache on a GPU: append, read back and attention against float64
numpy (kv4_ref)."""

import numpy as np
import pytest

import kv4_ref as ref
from gpu_util import device, say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32, BF16 = 0, 1
TYPES = {F32: torch.float32, BF16: torch.bfloat16}
HALF_STEP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def pages_of(n, hkv, hd, dev, fill=0xFF):
    """Pages whose every block reads as NaN until something is appended."""
    return torch.full((n, hkv, ref.block_bytes(hd)), fill, dtype=torch.uint8, device=dev)


def to(dev, a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev).to(dtype)


def ints(dev, a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).to(dev)


def vectors(rng, *shape):
    """Values as a cache meets them, some dims much larger; zero blocks, tiny ones, ties of the rounding."""
    x = rng.standard_normal(shape)
    x[..., 3::17] *= 8
    x = x.astype(np.float32)
    if shape[0] > 4:
        x[1, 0, :32] = 0
        x[2, 0, 32:64] *= 1e-38
        x[3, -1, :32] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5] * 4
        x[4, -1, 32:64] = -x[3, -1, :32] * 2.0 ** 40
    return x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hq, hkv, hd", [(4, 4, 64), (32, 8, 128), (7, 1, 64), (3, 3, 128), (32, 8, 64)])
@pytest.mark.parametrize("R, start", [(1, 0), (6, 11), (33, 5), (200, 131072)])
def test_append_and_read(dtype, hq, hkv, hd, R, start):
    from paper_2607_20507_amd import binding as B
    dev = device()
    say("append", dtype, hq, hkv, hd, R, start)
    rng = np.random.default_rng([hq, hd, R])
    P, theta = R // 16 + 4, 5e5
    assert B.spec_kv4_page_bytes(hkv, hd) == hkv * ref.block_bytes(hd)
    qkv = vectors(rng, R, hq + 2 * hkv, hd)
    pos = start + np.arange(R)
    table = rng.permutation(P)
    slot = table[(pos - start + start % 16) // 16] * 16 + pos % 16
    if R > 4:
        slot[[2, R - 1]] = [-1, 16 * P]  # padding rows: q alone
    kept = np.nonzero((slot >= 0) & (slot < 16 * P))[0]
    kp, vp = pages_of(P, hkv, hd, dev), pages_of(P, hkv, hd, dev)
    q = torch.empty(R, hq, hd, dtype=TYPES[dtype], device=dev)
    B.spec_op_rope_kv4(dtype, R, hq, hkv, hd, theta, to(dev, qkv), ints(dev, pos), ints(dev, slot), P, q, kp, vp)
    turned = ref.rotate(qkv[:, :hq + hkv].astype(np.float64), pos, theta)
    # q: fp64 angles rounded to fp32 (2^-24 each), two products and a sum in fp32 (3 roundings), one to dtype
    size = np.abs(qkv[:, :hq].astype(np.float64))
    size = size + np.roll(size, hd // 2, -1)
    err = np.abs(q.double().cpu().numpy() - turned[:, :hq])
    assert np.all(err <= HALF_STEP[dtype] * np.abs(turned[:, :hq]) * 1.01 + 4 * 2.0 ** -24 * size)
    # codes and scales: the whole of both pools, byte for byte
    want_k, want_v = (np.full((P, hkv, ref.block_bytes(hd)), 0xFF, np.uint8) for _ in range(2))
    ref.put(want_k, slot[kept], turned[kept, hq:].astype(np.float32).astype(np.float64), ref.k_place)
    ref.put(want_v, slot[kept], qkv[kept, hq + hkv:].astype(np.float64), ref.v_place)
    assert np.array_equal(kp.cpu().numpy(), want_k)
    assert np.array_equal(vp.cpu().numpy(), want_v)
    # read back: exact in both types; a slot outside the pool leaves its row alone; order and repeats are free
    order = np.concatenate([rng.permutation(R), [0, 0]])
    k, v = (torch.full((R + 2, hkv, hd), 7.0, dtype=TYPES[dtype], device=dev) for _ in range(2))
    B.spec_op_kv4_read(dtype, R + 2, hkv, hd, ints(dev, slot[order]), P, kp, vp, k, v)
    for got, pages, place in ((k, want_k, ref.k_place), (v, want_v, ref.v_place)):
        want = np.full((R + 2, hkv, hd), 7.0)
        inside = np.isin(order, kept)
        want[inside] = ref.get(pages, slot[order[inside]], hd, place)
        assert np.array_equal(got.double().cpu().numpy(), want)


@pytest.mark.parametrize("R, start", [(255, 0), (256, 7), (257, 0), (600, 1)])
def test_append_and_read_of_rows_spread_over_the_chip(R, start):
    """Whole rounds of 8 x 32 rows are taken in another order, the rows behind them are not."""
    test_append_and_read(BF16, 4, 2, 64, R, start)


def test_append_of_infinities_and_the_largest_values():
    from paper_2607_20507_amd import binding as B
    dev = device()
    hkv, hd, R = 2, 64, 3
    x = np.ones((R, 3 * hkv, hd), np.float32)
    x[0, 4, 3], x[1, 5, 40], x[2, 4, 0] = np.inf, np.nan, 2.0 ** 120
    kp, vp = pages_of(1, hkv, hd, dev, 0), pages_of(1, hkv, hd, dev, 0)
    q = torch.empty(R, hkv, hd, dtype=torch.bfloat16, device=dev)
    B.spec_op_rope_kv4(BF16, R, hkv, hkv, hd, 1e4, to(dev, x), ints(dev, [0, 1, 2]), ints(dev, [0, 5, 15]), 1, q, kp, vp)
    k, v = (torch.empty(R, hkv, hd, dtype=torch.float32, device=dev) for _ in range(2))
    B.spec_op_kv4_read(F32, R, hkv, hd, ints(dev, [0, 5, 15]), 1, kp, vp, k, v)
    assert np.array_equal(np.nan_to_num(v.cpu().numpy(), nan=-99.0), np.nan_to_num(ref.held(x[:, 4:]), nan=-99.0))
    assert bool(v[0, 0, :32].isnan().all()) and not bool(v[0, 0, 32:].isnan().any()) and not bool(k.isnan().any())


def cache(rng, lens, hkv, hd, dev, P=None, shared=False):
    """Pages, page table and fp64 values of sequences of the given lengths; everything else reads as NaN."""
    need = [(n + 15) // 16 for n in lens]
    P = P or sum(need) + 3
    if shared:
        first = rng.permutation(P)[:max(need)]
        table = np.tile(first, (len(lens), 1))
    else:
        perm = rng.permutation(P)
        table = np.full((len(lens), max(max(need), 1)), -1)
        for i, o in enumerate(np.cumsum(need) - need):
            table[i, :need[i]] = perm[o:o + need[i]]
    k_np, v_np = (np.full((P, hkv, ref.block_bytes(hd)), 0xFF, np.uint8) for _ in range(2))
    values = []
    for i, n in enumerate(lens):
        if shared and i and n <= len(values[0][0]):
            values.append([x[:n] for x in values[0]])
            continue
        slot = table[i][np.arange(n) // 16] * 16 + np.arange(n) % 16
        kv = []
        for pages, place in ((k_np, ref.k_place), (v_np, ref.v_place)):
            x = vectors(rng, n, hkv, hd).astype(np.float64) if n else np.zeros((0, hkv, hd))
            put_fast(pages, slot, x, place)
            kv.append(ref.held(x) if n < 300 else ref.get(pages, slot, hd, place))
        values.append(kv)
    return ints(dev, table).cpu().numpy(), to(dev, k_np, torch.uint8), to(dev, v_np, torch.uint8), values


def put_fast(pages, slot, x, place):
    """ref.put, over all rows of a token offset at once."""
    hd = x.shape[-1]
    if len(x) < 300:
        return ref.put(pages, slot, x, place)
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(b).max(-1)
    with np.errstate(divide="ignore"):
        e = np.maximum(np.where(top > 0, np.ceil(np.log2(top / 6)), -126), -126).astype(int)  # (any scale makes a valid page)
    r = np.minimum(np.abs(b) * 2.0 ** -e[..., None].astype(float), 6)
    code = np.abs(r[..., None] - ref.LEVELS).argmin(-1) + 8 * np.signbit(b)
    code, e = code.reshape(x.shape), e + 127
    for t in range(16):
        rows = np.nonzero(slot % 16 == t)[0]
        at = slot[rows] // 16
        for d in range(hd):
            byte, nib, sb = place(t, d, hd)
            pages[at, :, byte] = (pages[at, :, byte] & (0xF0 if nib == 0 else 0x0F)) | (code[rows, :, d] << (4 * nib)).astype(np.uint8)
            pages[at, :, sb] = e[rows, :, d // 32]


def attend(dtype, rows, pos0, table, P, hq, hkv, hd, q, kp, vp, dev, stream=None):
    from paper_2607_20507_amd import binding as B
    nb = B.spec_op_attention_kv4_workspace_bytes(dtype, rows, pos0, table.shape[1], hq, hkv, hd)
    ws = torch.full((nb + 256,), 0xFF, dtype=torch.uint8, device=dev)
    out = torch.full((sum(rows) + 1, hq * hd), 7.0, dtype=TYPES[dtype], device=dev)
    B.spec_op_attention_kv4(dtype, rows, pos0, table, P, hq, hkv, hd, q, kp, vp, out[:-1], ws[:nb], stream)
    assert bool((ws[nb:] == 0xFF).all()) and bool((out[-1] == 7.0).all())  # nothing beyond the workspace and the rows
    return out[:-1]


def check(dtype, rows, pos0, hq, hkv, hd, dev, seed=0, only=None, shared=False):
    rng = np.random.default_rng([seed, hq, hd, len(rows)])
    table, kp, vp, values = cache(rng, [r + p for r, p in zip(rows, pos0)], hkv, hd, dev, shared=shared)
    q = to(dev, vectors(rng, sum(rows), hq, hd) / 4, TYPES[dtype])
    got = attend(dtype, rows, pos0, table, kp.shape[0], hq, hkv, hd, q, kp, vp, dev)
    got = got.double().cpu().numpy().reshape(-1, hq, hd)
    q64, r0 = q.double().cpu().numpy(), 0
    for i, (r, p) in enumerate(zip(rows, pos0)):
        if r and (only is None or i in only):
            k, v = values[i]
            want, mag, big = ref.attention(q64[r0:r0 + r], k, v, p)
            # scores: q k in fp32, a sum of hd products of which each adds a rounding: hd 2^-24 sum |q k| / sqrt(hd),
            # one more for the scale and the difference to the maximum (|s| <= big each), which is a relative error
            # of p and of its sum; p itself: exp2 (2^-22), its rounding to dtype, sums over n keys in fp32
            n = len(k)
            score = (hd + 4) * 2.0 ** -24 * big
            rel = 2 * score + 2.0 ** -22 + HALF_STEP[dtype] + (n / 32 + 40) * 2.0 ** -24
            tol = rel * (mag + np.abs(want)) + HALF_STEP[dtype] * np.abs(want)
            err = np.abs(got[r0:r0 + r] - want)
            assert np.all(err <= tol), (i, float((err / tol).max()))
        r0 += r


HEADS = [(F32, 4, 4, 64), (F32, 8, 2, 128), (F32, 32, 1, 64), (BF16, 16, 16, 64), (BF16, 32, 8, 128), (BF16, 32, 8, 64),
         (BF16, 7, 1, 64), (BF16, 6, 2, 128), (BF16, 16, 1, 128), (BF16, 64, 1, 64)]


@pytest.mark.parametrize("dtype, hq, hkv, hd", HEADS)
@pytest.mark.parametrize("rows, pos0", [
    ([1], [0]), ([1], [15]), ([2], [31]), ([6], [500]), ([3, 0, 8, 1], [0, 40, 29, 128]), ([17, 5], [3, 640]), ([0, 1], [9, 2])])
def test_attention(dtype, hq, hkv, hd, rows, pos0):
    dev = device()
    say("attention", dtype, hq, hkv, hd, rows, pos0)
    check(dtype, rows, pos0, hq, hkv, hd, dev)


@pytest.mark.parametrize("dtype, hq, hkv, hd", [(F32, 4, 4, 64), (BF16, 8, 2, 128), (BF16, 4, 2, 64), (BF16, 7, 1, 64)])
@pytest.mark.parametrize("rows, pos0", [([63], [5]), ([64], [0]), ([70, 130], [0, 33]), ([300], [100]), ([64, 0, 65], [400, 3, 0])])
def test_attention_of_prompts(dtype, hq, hkv, hd, rows, pos0):
    dev = device()
    say("prompt attention", dtype, hq, hkv, hd, rows, pos0)
    check(dtype, rows, pos0, hq, hkv, hd, dev, seed=1)


def test_long_context_is_split():
    dev = device()
    check(BF16, [1], [9000], 8, 2, 128, dev, seed=2)
    check(F32, [2], [5000], 4, 4, 64, dev, seed=2)


def test_items_of_more_keys_than_staged_page_ids():
    """16 sequences over one long prefix: a work item walks more than 4096 keys."""
    dev = device()
    n = 16
    pos0 = [20000 - 37 * i for i in range(n)]
    check(BF16, [2] * n, pos0, 32, 8, 64, dev, seed=3, only=(0, 15), shared=True)


def test_a_prefix_shared_by_sequences():
    dev = device()
    check(BF16, [5, 5, 64], [100, 99, 41], 8, 2, 128, dev, seed=4, shared=True)


def test_pages_beyond_32_bit_offsets():
    from paper_2607_20507_amd import binding as B
    dev = device()
    hkv, hd, P = 8, 128, 520000  # 4.5 GB of keys
    rng = np.random.default_rng(9)
    kp, vp = pages_of(P, hkv, hd, dev), pages_of(P, hkv, hd, dev)
    R = 20
    x = vectors(rng, R, 3 * hkv, hd)
    slot = np.where(np.arange(R) < 16, (P - 1) * 16, 3 * 16) + np.arange(R) % 16
    q = torch.empty(R, hkv, hd, dtype=torch.bfloat16, device=dev)
    B.spec_op_rope_kv4(BF16, R, hkv, hkv, hd, 1e4, to(dev, x), ints(dev, np.arange(R)), ints(dev, slot), P, q, kp, vp)
    k, v = (torch.empty(R, hkv, hd, dtype=torch.bfloat16, device=dev) for _ in range(2))
    B.spec_op_kv4_read(BF16, R, hkv, hd, ints(dev, slot), P, kp, vp, k, v)
    assert np.array_equal(v.double().cpu().numpy(), ref.held(x[:, 2 * hkv:]))
    k64, v64 = k.double().cpu().numpy(), v.double().cpu().numpy()
    out = attend(BF16, [R], [0], np.array([[P - 1, 3]], np.int32), P, hkv, hkv, hd, q, kp, vp, dev).double().cpu().numpy()
    want, mag, big = ref.attention(q.double().cpu().numpy(), k64, v64, 0)
    tol = (2.0 ** -7 + 2 * (hd + 4) * 2.0 ** -24 * big) * (mag + np.abs(want))
    assert np.all(np.abs(out.reshape(want.shape) - want) <= tol)


def test_a_row_of_nan_stays_in_its_sequence():
    dev = device()
    hq, hkv, hd = 8, 2, 64
    rng = np.random.default_rng(11)
    table, kp, vp, values = cache(rng, [40, 50], hkv, hd, dev)
    page = int(table[0, 1])
    kp[page] = 0xFF  # keys 16 .. 31 of sequence 0
    q = to(dev, vectors(rng, 8, hq, hd), torch.bfloat16)
    out = attend(BF16, [4, 4], [36, 46], table, kp.shape[0], hq, hkv, hd, q, kp, vp, dev)
    assert bool(out[:4].isnan().all()) and not bool(out[4:].isnan().any())


def test_attention_captured_and_replayed_on_another_stream():
    from paper_2607_20507_amd import binding as B
    dev = device()
    hq, hkv, hd, rows, pos0 = 32, 8, 128, [6], [2047]
    rng = np.random.default_rng(12)
    table, kp, vp, _ = cache(rng, [2053], hkv, hd, dev)
    q = torch.empty(6, hq, hd, dtype=torch.bfloat16, device=dev)
    nb = B.spec_op_attention_kv4_workspace_bytes(BF16, rows, pos0, table.shape[1], hq, hkv, hd)
    ws = torch.empty(nb, dtype=torch.uint8, device=dev)
    out = torch.empty(6, hq * hd, dtype=torch.bfloat16, device=dev)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        try:
            B.spec_op_attention_kv4(BF16, rows, pos0, table, kp.shape[0], hq, hkv, hd, q, kp, vp, out, ws, side)
            taken = True
        except B.SpecError as e:  # tables beyond what a captured call takes
            assert e.status == B.SPEC_E_UNSUPPORTED
            taken = False
            out.zero_()
    for seed in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator(device=dev).manual_seed(seed), device=dev))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if taken:
            eager = attend(BF16, rows, pos0, table, kp.shape[0], hq, hkv, hd, q, kp, vp, dev)
            assert torch.equal(out, eager), seed
    short = [100]
    table1 = table[:, :7].copy()
    nb = B.spec_op_attention_kv4_workspace_bytes(BF16, [1], short, 7, hq, hkv, hd)
    ws1 = torch.empty(nb, dtype=torch.uint8, device=dev)
    out1 = torch.empty(1, hq * hd, dtype=torch.bfloat16, device=dev)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.spec_op_attention_kv4(BF16, [1], short, table1, kp.shape[0], hq, hkv, hd, q[:1], kp, vp, out1, ws1, side)
    for seed in range(4):
        q.copy_(torch.randn(q.shape, generator=torch.Generator(device=dev).manual_seed(seed), device=dev))
        ws1.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = attend(BF16, [1], short, table1, kp.shape[0], hq, hkv, hd, q[:1], kp, vp, dev)
        assert torch.equal(out1, eager), seed
