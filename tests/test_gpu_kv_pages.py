"""spec_op_kv_copy_pages: page copies in every plane of a pool, on a GPU."""

import numpy as np
import pytest

from gpu_util import device, say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def workspace(B, n, dev):
    return torch.empty(max(256, B.spec_op_kv_copy_pages_workspace_bytes(n)), dtype=torch.uint8, device=dev)


@pytest.mark.parametrize("planes, pages, page, n, copies", [
    (1, 2, 16, 1, 1), (3, 7, 48, 2, 2), (4, 40, 2176, 5, 3), (2, 900, 16384 + 16, 400, 1), (24, 64, 32768, 8, 4), (2, 5000, 544, 100, 20)])
def test_copies(planes, pages, page, n, copies):
    from paper_2607_20507_amd import binding as B
    dev = device()
    say("copy pages", planes, pages, page, n, copies)
    rng = np.random.default_rng([planes, pages, n])
    pool = torch.randint(0, 256, (planes, pages, page), dtype=torch.uint8, device=dev)
    perm = rng.permutation(pages)
    src, dst = np.tile(perm[:n], copies)[:pages - n], perm[n:n + min(n * copies, pages - n)]
    want = pool.clone()
    want[:, torch.from_numpy(dst).to(dev)] = pool[:, torch.from_numpy(src).to(dev)]
    B.spec_op_kv_copy_pages(pool, src, dst, workspace(B, len(src), dev))
    assert torch.equal(pool, want)  # the other pages are as they were


def test_refused_calls_change_nothing():
    from paper_2607_20507_amd import binding as B
    dev = device()
    pool = torch.randint(0, 256, (2, 8, 64), dtype=torch.uint8, device=dev)
    before = pool.clone()
    for src, dst in (([1, 2], [3, 3]), ([1, 2], [2, 3]), ([1], [8]), ([-1], [1])):
        with pytest.raises(B.SpecError):
            B.spec_op_kv_copy_pages(pool, src, dst, workspace(B, 2, dev))
    torch.cuda.synchronize()
    assert torch.equal(pool, before)


def test_pages_beyond_32_bit_offsets():
    from paper_2607_20507_amd import binding as B
    dev = device()
    pages, page = 140000, 32768  # 4.6 GB a plane
    pool = torch.zeros(2, pages, page, dtype=torch.uint8, device=dev)
    g = torch.Generator(device=dev).manual_seed(2)
    for p in (5, pages - 3):
        pool[:, p] = torch.randint(0, 256, (2, page), dtype=torch.uint8, generator=g, device=dev)
    B.spec_op_kv_copy_pages(pool, [5, pages - 3], [pages - 1, 6], workspace(B, 2, dev))
    assert torch.equal(pool[:, pages - 1], pool[:, 5]) and torch.equal(pool[:, 6], pool[:, pages - 3])
    assert not pool[:, pages - 2].any() and not pool[:, 7].any()


def test_captured_and_replayed():
    from paper_2607_20507_amd import binding as B
    dev = device()
    pool = torch.zeros(3, 32, 4352, dtype=torch.uint8, device=dev)
    src, dst = [1, 2, 1], [9, 30, 11]
    ws = workspace(B, 3, dev)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        B.spec_op_kv_copy_pages(pool, src, dst, ws, side)
    for seed in range(4):
        pool.copy_(torch.randint(0, 256, pool.shape, dtype=torch.uint8, device=dev))
        want = pool.clone()
        want[:, dst] = pool[:, src]
        ws.random_(0, 256)  # a replay brings its own tables
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool, want), seed


def test_capture_of_large_tables_is_refused():
    from paper_2607_20507_amd import binding as B
    dev = device()
    pool = torch.zeros(1, 2000, 16, dtype=torch.uint8, device=dev)
    ws = workspace(B, 900, dev)
    marker = torch.zeros(4, device=dev)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        marker.add_(1)
        with pytest.raises(B.SpecError) as e:
            B.spec_op_kv_copy_pages(pool, np.arange(900), np.arange(900, 1800), ws, side)
        assert e.value.status == B.SPEC_E_UNSUPPORTED
    graph.replay()
    torch.cuda.synchronize()
    assert float(marker.sum()) == 4.0
