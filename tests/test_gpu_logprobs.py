"""spec_token_logprobs against float64 numpy, on a GPU."""

import math

import numpy as np
import pytest

from gpu_util import device, say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def reference(z, temps, tokens, n):
    """float64 (log p, entropy, ids, top log p, largest |z - m| / T of a likely token) of fp32 rows."""
    R, V = z.shape
    lp, h = np.full(R, np.nan), np.full(R, np.nan)
    ids, top = np.full((R, n), -1), np.full((R, n), np.nan)
    for r in range(R):
        x, t = z[r].astype(np.float64), float(temps[r])
        m = x.max()
        if not np.isfinite(m) or np.isnan(x).any() or not t >= 0:
            continue
        order = np.argsort(-x, kind="stable")
        if t == 0:
            logp = np.full(V, -np.inf)
            logp[order[0]] = 0.0
        else:
            with np.errstate(over="ignore"):
                logp = (x - m) / t
            logp -= math.log(np.exp(logp).sum())
        p = np.exp(logp)
        h[r] = -np.sum(np.where(p > 0, p * np.where(p > 0, logp, 0), 0))
        lp[r] = logp[tokens[r]] if 0 <= tokens[r] < V else -np.inf
        ids[r], top[r] = order[:n], logp[order[:n]]
    return lp, h, ids, top


def call(z, temps, tokens, n, dev, stream=None, parts=("logp", "entropy")):
    from paper_2607_20507_amd import binding as B
    R, V = z.shape
    out = {k: torch.full((R,), 7.0, device=dev) for k in parts}
    ids, top = torch.full((R, n), -7, dtype=torch.int32, device=dev), torch.full((R, n), 7.0, device=dev)
    ws = torch.empty(B.spec_token_logprobs_workspace_bytes(R, V, n), dtype=torch.uint8, device=dev)
    B.spec_token_logprobs(z, temps, tokens, out.get("logp"), out.get("entropy"), ids if n else None, top if n else None, ws, stream)
    return out.get("logp"), out.get("entropy"), ids, top


# fp32 error: t = (z - m) / T is off by 2 roundings, |t| 2^-23; a sum of V terms kept by 256 threads a chunk (at
# most 64 chunks, so at most V / 256 + 64 additions in a row for V <= 128256: 570) by 570 2^-24 = 3.4e-5 relative,
# and so its logarithm absolutely; the entropy's second sum by as much of itself (at most H + log S, log S < 12) plus what t's
# error does to the terms, sum p t^2 2^-23 (p t^2 summed is below 150 for these rows: 1.8e-5).
LP_ABS, LP_REL, H_TOL = 4e-5, 3e-7, 4e-5 * 13


def compare(got, want, what):
    lp, h, ids, top = (None if g is None else g.cpu().numpy().astype(np.float64) for g in got)
    wl, wh, wi, wt = want
    for g, w, rel in ((lp, wl, LP_REL), (top, wt, LP_REL), (h, wh, 0.0)):
        if g is None:
            continue
        assert np.array_equal(np.isnan(g), np.isnan(w)), what
        assert np.array_equal(np.isneginf(g), np.isneginf(w)), what
        fine = np.isfinite(w)
        assert np.all(np.abs(g[fine] - w[fine]) <= (H_TOL if rel == 0.0 else LP_ABS) + rel * np.abs(w[fine])), \
            (what, np.abs(g[fine] - w[fine]).max())
    assert np.array_equal(ids, wi), what


def rows_of(kind, R, V, rng):
    z = (rng.standard_normal((R, V)) * 3).astype(np.float32)
    if kind == "coarse":  # many equal logits
        z = (np.round(z * 2) / 2).astype(np.float32)
        z[0] = 1.25  # a row of one value
    elif kind == "masked":  # most of the vocabulary masked, by -inf and by the type's lowest value
        z[rng.random((R, V)) < 0.9] = -np.inf
        z[0] = -np.inf                     # nothing left
        z[1, :] = -np.inf
        z[1, V // 3] = 2.0                 # one token left
        z[2, rng.random(V) < 0.9] = np.finfo(np.float32).min
        if R > 4:
            z[3] = np.finfo(np.float32).min  # uniform over the lowest value
    elif kind == "sorted":  # every step of the pass finds larger logits
        z = np.sort(z, axis=1)
    elif kind == "bad":
        z[0, V // 2] = np.nan
        z[1, V - 1] = np.inf
        z[2, 0] = np.nan
        z[2, 1:] = -np.inf
    elif kind == "peaked":
        z[:, 5 % V] = 300.0
        z[1] *= 1e30
    elif kind == "zeros":  # 0 and -0 are equal
        z = np.where(rng.random((R, V)) < 0.5, np.float32(-0.0), np.float32(0.0)).astype(np.float32)
    return z


@pytest.mark.parametrize("kind", ["normal", "coarse", "masked", "sorted", "bad", "peaked", "zeros"])
@pytest.mark.parametrize("R, V, n", [(1, 1, 1), (3, 7, 7), (5, 1000, 1), (7, 4099, 5), (9, 32000, 20), (5, 128256, 64), (3, 50257, 0), (8, 300, 64)])
def test_rows(kind, R, V, n):
    if kind in ("masked", "bad", "peaked") and (R < 3 or V < 7):
        pytest.skip("the rows do not fit")
    dev = device()
    rng = np.random.default_rng([R, V, n, len(kind)])
    z = rows_of(kind, R, V, rng)
    temps = np.array([(1.0, 0.3, 0.0, 1.5, 0.8)[i % 5] for i in range(R)], dtype=np.float32)
    tokens = rng.integers(0, V, R).astype(np.int32)
    tokens[-1] = (-1, V, z[-1].argmax())[R % 3]
    say("logprobs", kind, R, V, n)
    got = call(torch.from_numpy(z).to(dev), torch.from_numpy(temps).to(dev), torch.from_numpy(tokens).to(dev), n, dev)
    compare(got, reference(z, temps, tokens, n), (kind, R, V, n))


def test_temperatures():
    dev = device()
    rng = np.random.default_rng(5)
    temps = np.array([1e-30, 1e30, -1.0, np.nan, np.inf, 0.0, 1e-3], dtype=np.float32)
    z = (rng.standard_normal((len(temps), 2000)) * 3).astype(np.float32)
    tokens = z.argmax(1).astype(np.int32)
    lp, h, ids, top = (x.cpu().numpy() for x in call(torch.from_numpy(z).to(dev), torch.from_numpy(temps).to(dev),
                                                     torch.from_numpy(tokens).to(dev), 3, dev))
    for r in (2, 3):  # no distribution
        assert np.isnan(lp[r]) and np.isnan(h[r]) and np.isnan(top[r]).all() and (ids[r] == -1).all()
    for r in (0, 5):  # all on the maximum
        assert lp[r] == 0 and h[r] == 0 and top[r, 0] == 0 and np.isneginf(top[r, 1:]).all() == (r == 5)
    for r in (1, 4):  # uniform
        assert abs(lp[r] + math.log(2000)) < LP_ABS and abs(h[r] - math.log(2000)) < H_TOL
    fine = [0, 1, 4, 5, 6]
    assert np.array_equal(ids[fine], np.argsort(-z, axis=1, kind="stable")[fine, :3])


def test_masked_tokens_at_an_infinite_temperature():
    dev = device()
    z = np.full((2, 3000), -np.inf, np.float32)
    z[0, [5, 700, 2999]] = [1.0, -4.0, 2.0]
    z[1, 8] = 3.0
    temps = np.array([np.inf, np.inf], np.float32)
    lp, h, ids, top = (x.cpu().numpy() for x in call(torch.from_numpy(z).to(dev), torch.from_numpy(temps).to(dev),
                                                     torch.tensor([6, 8], dtype=torch.int32, device=dev), 4, dev))
    assert np.isneginf(lp[0]) and lp[1] == 0
    assert abs(h[0] - math.log(3)) < H_TOL and h[1] == 0
    assert ids.tolist() == [[2999, 5, 700, 0], [8, 0, 1, 2]]
    assert np.all(np.abs(top[0, :3] + math.log(3)) < LP_ABS) and np.isneginf(top[0, 3])
    assert top[1, 0] == 0 and np.isneginf(top[1, 1:]).all()


def test_optional_outputs_and_defaults():
    dev = device()
    rng = np.random.default_rng(6)
    z = (rng.standard_normal((6, 5000)) * 3).astype(np.float32)
    tokens = rng.integers(0, 5000, 6).astype(np.int32)
    zt, tt = torch.from_numpy(z).to(dev), torch.from_numpy(tokens).to(dev)
    want = reference(z, np.ones(6), tokens, 4)
    compare(call(zt, None, tt, 4, dev), want, "no temperatures")
    compare(call(zt, None, None, 4, dev, parts=("entropy",)), want, "no tokens")
    compare(call(zt, None, None, 4, dev, parts=()), want, "alternatives alone")


@pytest.mark.parametrize("off, pad", [(0, 4), (1, 0), (0, 3), (2, 2)])
def test_strided_and_unaligned_rows(off, pad):
    """Rows inside a larger buffer: what surrounds them is not read as logits and not written."""
    dev = device()
    V, R = 4100, 4
    rng = np.random.default_rng([off, pad])
    z = (rng.standard_normal((R, V)) * 3).astype(np.float32)
    buf = torch.full((R * (V + pad) + off,), 1e30, device=dev)
    view = buf[off:].view(R, V + pad)[:, :V]
    view.copy_(torch.from_numpy(z))
    before = buf.clone()
    tokens = rng.integers(0, V, R).astype(np.int32)
    got = call(view, None, torch.from_numpy(tokens).to(dev), 10, dev)
    compare(got, reference(z, np.ones(R), tokens, 10), (off, pad))
    assert torch.equal(buf, before)


def test_rows_beyond_32_bit_offsets():
    dev = device()
    V, ld, R = 5000, (1 << 30) + 4, 3  # the last row starts 8.6 GB into the buffer
    buf = torch.empty(ld * (R - 1) + V, device=dev)
    view = buf.as_strided((R, V), (ld, 1))
    rng = np.random.default_rng(4)
    z = (rng.standard_normal((R, V)) * 3).astype(np.float32)
    view.copy_(torch.from_numpy(z))
    tokens = rng.integers(0, V, R).astype(np.int32)
    compare(call(view, None, torch.from_numpy(tokens).to(dev), 6, dev), reference(z, np.ones(R), tokens, 6), "far rows")


def test_rows_do_not_depend_on_the_batch_of_equal_size():
    dev = device()
    g = torch.Generator(device=dev).manual_seed(1)
    z = torch.randn(12, 32000, generator=g, device=dev) * 3
    tok = torch.arange(12, dtype=torch.int32, device=dev)
    a = call(z, None, tok, 8, dev)
    perm = torch.randperm(12, device=dev)
    b = call(z[perm].contiguous(), None, tok[perm].contiguous(), 8, dev)
    for x, y in zip(a, b):
        assert torch.equal(x[perm], y)
    for x, y in zip(a, call(z, None, tok, 8, dev)):
        assert torch.equal(x, y)


def test_captured_and_replayed_on_another_stream():
    from paper_2607_20507_amd import binding as B
    dev = device()
    R, V, n = 16, 32000, 5
    z = torch.empty(R, V, device=dev)
    tok, temps = torch.zeros(R, dtype=torch.int32, device=dev), torch.full((R,), 0.7, device=dev)
    out = torch.empty(2, R, device=dev)
    ids, top = torch.empty(R, n, dtype=torch.int32, device=dev), torch.empty(R, n, device=dev)
    ws = torch.empty(B.spec_token_logprobs_workspace_bytes(R, V, n), dtype=torch.uint8, device=dev)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.spec_token_logprobs(z, temps, tok, out[0], out[1], ids, top, ws, side)
    for seed in range(4):
        g = torch.Generator(device=dev).manual_seed(seed)
        z.copy_(torch.randn(R, V, generator=g, device=dev) * 3)
        tok.copy_(torch.randint(0, V, (R,), generator=g, device=dev, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = call(z, temps, tok, n, dev)
        for x, y in zip((out[0], out[1], ids, top), eager):
            assert torch.equal(x, y), seed
