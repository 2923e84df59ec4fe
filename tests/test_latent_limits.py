"""CPU checks: attention over a latent cache refuses, before anything is enqueued, what makes more workgroups than a launch
holds (a launch counts its threads in 32 bits)."""

import os

import numpy as np
import pytest

from paper_2607_20507_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

P = 0x1000  # an address that no refused call may touch


def sized(dtype, rows, pos0, H, rank, max_pages):
    return B.lib().spec_op_attention_latent_workspace_bytes(dtype, len(rows), rows.ctypes.data, pos0.ctypes.data, max_pages, H, 64, 32, rank, 64)


def attention(dtype, rows, pos0, H, rank, max_pages):
    table = np.zeros((len(rows), max_pages), np.int32)
    return B.lib().spec_op_attention_latent(dtype, len(rows), rows.ctypes.data, pos0.ctypes.data, table.ctypes.data, max_pages, 1, H, 64, 32, rank,
                                            64, 0.1, P, P, P, 64 * rank, P, 64 * rank, P, P, (1 << 63) - 1, None)


# workgroups of fp32 take 16 rows x heads of a sequence: 512 threads at rank 256, 256 at rank 512
@pytest.mark.parametrize("rank, seqs, rows, H", [
    (256, 1, 1 << 24, 8),       # 2^23 tiles of one sequence
    (256, 1 << 23, 1, 1),       # one of each of 2^23 sequences
    (512, 1, 1 << 25, 8)])      # 2^24 tiles
def test_more_workgroups_than_a_launch_holds(rank, seqs, rows, H):
    r, p = np.full(seqs, rows, np.int32), np.zeros(seqs, np.int32)
    pages = (rows + 15) // 16
    assert sized(B.SPEC_F32, r, p, H, rank, pages) == 0
    assert attention(B.SPEC_F32, r, p, H, rank, pages) == B.SPEC_E_UNSUPPORTED
    assert "spec_op_attention_latent: more workgroups than a launch holds" in B.lib().spec_last_error(None).decode()


def test_the_most_that_a_launch_holds_is_sized():
    """2^23 - 1 workgroups of 512 threads; 2^23 and more of 256."""
    r, p = np.full(1, (1 << 24) - 2, np.int32), np.zeros(1, np.int32)
    rows, lat = int(r[0]), 8 * 256 * 4
    assert sized(B.SPEC_F32, r, p, 8, 256, 1 << 20) >= 2 * rows * lat
    r[0] = 1 << 24
    assert sized(B.SPEC_F32, r, p, 8, 512, 1 << 20) >= 4 * rows * lat
