"""What a rollback leaves in the pools, at lengths that end a page and at others:
every position from the new length on that no other sequence holds reads as
zeros in every layer, K and V, of both caches; kept positions and pages that
other sequences hold are as they were."""

import numpy as np
import pytest

from test_gpu_kv_clear import _Pool, _session, _slot
from tests.gpu_util import say, torch
from workloads import uniform_prompts

pytestmark = pytest.mark.gpu


def _pools(gpu, cfg, layers, npages):
    torch.cuda.synchronize()
    return (_Pool(gpu.kv_target, cfg.target, layers[0], npages), _Pool(gpu.kv_draft, cfg.draft, layers[1], npages))


@pytest.mark.parametrize("which", ["fp32", "bf16"])
@pytest.mark.parametrize("new_len", [0, 16, 17, 31, 32, 48])
def test_alone(which, new_len):
    gpu, cfg, layers, npages = _session(which, 2)
    prompts = uniform_prompts(cfg.seed + 21, [57, 41], cfg.target.vocab)
    say("rollback", which, "to", new_len)
    gpu.prefill([1, 2], prompts)
    before, info = _pools(gpu, cfg, layers, npages), gpu.seq_info(1)
    gpu.rollback(1, new_len)
    after, other = _pools(gpu, cfg, layers, npages), gpu.seq_info(2)
    for b, a, side in zip(before, after, ("target", "draft")):
        pages = info[f"pages_{side}"]
        for pos in range(info[f"{side}_len"]):
            was, now = b.token_bits(*_slot(pages, pos)), a.token_bits(*_slot(pages, pos))
            assert was.any()
            if pos < new_len:
                assert np.array_equal(was, now), (side, pos, "kept position changed")
            else:
                assert not now.any(), (side, pos, "not cleared")
        for pos in range(other[f"{side}_len"]):
            at = _slot(other[f"pages_{side}"], pos)
            assert np.array_equal(b.token_bits(*at), a.token_bits(*at)), (side, pos, "another sequence's")
    gpu.close()


@pytest.mark.parametrize("which", ["fp32", "bf16"])
@pytest.mark.parametrize("new_len", [0, 16, 20, 32, 48, 50])
def test_with_shared_pages(which, new_len):
    gpu, cfg, layers, npages = _session(which, 2)
    prompt = uniform_prompts(cfg.seed + 22, [57], cfg.target.vocab)[0]
    gpu.prefill([1], [prompt])
    gpu.fork(1, [2])
    info = gpu.seq_info(2)
    shared = info["target_len"] // 16
    before = _pools(gpu, cfg, layers, npages)
    say("rollback of a fork", which, "to", new_len)
    gpu.rollback(2, new_len)
    after, left, first = _pools(gpu, cfg, layers, npages), gpu.seq_info(2), gpu.seq_info(1)
    for b, a, side in zip(before, after, ("target", "draft")):
        for pos in range(first[f"{side}_len"]):
            at = _slot(first[f"pages_{side}"], pos)
            assert np.array_equal(b.token_bits(*at), a.token_bits(*at)), (side, pos, "another sequence's")
        pages = left[f"pages_{side}"]
        for pos in range(16 * len(pages)):  # what it kept, with a copy of a shared last page
            now = a.token_bits(*_slot(pages, pos))
            if pos < new_len:
                assert np.array_equal(now, b.token_bits(*_slot(info[f"pages_{side}"], pos))), (side, pos, "kept position changed")
            else:
                assert not now.any(), (side, pos, "not cleared")
        own = info[f"pages_{side}"][shared]  # the fork's own last page, given up or cleared from new_len on
        if own not in pages:
            for off in range(16):
                assert not a.token_bits(own, off).any(), (side, off, "given up uncleared")
    gpu.close()
