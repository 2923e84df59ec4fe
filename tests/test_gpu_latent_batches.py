"""Attention over a latent cache: workspaces that held other calls' values, sequences alone and among others, and entries that
are not finite in every tile."""

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


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_workspace_that_held_other_calls(dtype):
    """Calls of both forms, of every tile, with parts and without, take turns in one workspace: each gives the bits that it gives in
    one of its own, where nothing but NaN stood."""
    device()
    batches = [([6, 1, 400, 4], [1500, 20, 700, 333], 16, SMALL), ([1], [9000], 16, BIG), ([1, 1], [40, 3000], 32, SMALL),
               ([300], [2000], 4, BIG), ([8] * 60, [300] * 60, 16, SMALL), ([2, 1], [100, 17], 3, BIG)]
    cases = [L.Case(dtype, rows, pos0, H, seed=30 + i, **sizes) for i, (rows, pos0, H, sizes) in enumerate(batches)]
    want = []
    for c, b in zip(cases, batches):
        say("own workspace", dtype, *b)
        want.append(c.run(B).clone())
        assert torch.isfinite(want[-1]).all() and L.row_error(want[-1], c.ref()) <= L.TOL[dtype]
    ws = torch.full((max(c.workspace(B).numel() for c in cases),), 0xFF, dtype=torch.uint8, device="cuda")
    for order in (range(6), reversed(range(6)), [3, 0, 3, 1, 5, 1, 4, 2, 4]):
        for i in order:
            say("shared workspace", dtype, i)
            cases[i].out.fill_(7)
            assert torch.equal(cases[i].run(B, ws), want[i])
            assert (cases[i].out[len(cases[i].q):] == 7).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sizes", [BIG, SMALL], ids=["512", "256"])
def test_a_sequence_alone_and_among_others(dtype, sizes):
    """The same rows, alone and in batches that change their tiles, parts and order: the same answer but for roundings."""
    device()
    rows, pos0, H = [3, 1, 40, 7, 1], [2500, 900, 60, 0, 31], 8
    whole = L.Case(dtype, rows, pos0, H, seed=41, **sizes)
    ref, first = whole.ref(), np.cumsum([0] + rows)

    def part(seqs):
        c = L.Case(dtype, [rows[i] for i in seqs], [pos0[i] for i in seqs], H, seed=0, **sizes)
        c.P, c.pages, c.w_k, c.w_v = whole.P, whole.pages, whole.w_k, whole.w_v
        c.table = whole.table[seqs].copy()
        at = np.concatenate([np.arange(first[i], first[i + 1]) for i in seqs])
        c.q = whole.q[torch.from_numpy(at).to("cuda")].contiguous()
        return c, ref[torch.from_numpy(at).to("cuda")]

    for seqs in ([0, 1, 2, 3, 4], [0], [1], [2], [3], [4], [4, 2, 0], [1, 0], [3, 2, 1, 0, 4]):
        say("sequences", dtype, sizes, seqs)
        c, want = part(seqs)
        got = c.run(B)
        assert torch.isfinite(got).all() and L.row_error(got, want) <= L.TOL[dtype]


# heads and rows of one sequence: in bf16 tiles of 16 (whole rows of it, or a row's heads), 32 and 64, and the second form; whole
# contexts and parts; a context that ends inside a chunk of 32 keys, where a single row's own key is in a chunk that is cleaned
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("sizes", [BIG, SMALL], ids=["512", "256"])
@pytest.mark.parametrize("rows, H", [(4, 4), (16, 1), (1, 16), (2, 16), (8, 4), (5, 12), (30, 3)])
@pytest.mark.parametrize("pos0", [70, 2500])
def test_entries_that_are_not_finite(dtype, sizes, rows, H, pos0):
    device()
    rank = sizes["rank"]
    c = L.Case(dtype, [rows, 1], [pos0, 31], H, seed=50, **sizes)
    flat, slots = c.pages.view(-1, rank + sizes["rope"]), c.slots(0)
    whole = flat.clone()
    for bad in sorted({0, rows // 2, rows - 1}):
        for dim, value in [(0, math.nan), (rank - 1, math.inf), (rank // 2 + 5, -math.inf), (rank + 3, math.nan)]:
            say("not finite", dtype, sizes, rows, H, pos0, bad, dim, value)
            flat.copy_(whole)
            flat[slots[pos0 + bad], dim] = value  # the key of row `bad`
            got, ref = c.run(B), c.ref()
            fine = torch.isfinite(ref).all(-1)
            assert fine[:bad].all() and not fine[bad:rows].any() and fine[rows:].all()
            assert torch.isfinite(got[fine]).all() and L.row_error(got[fine], ref[fine]) <= L.TOL[dtype]
            assert not torch.isfinite(got[~fine]).all(-1).any()
