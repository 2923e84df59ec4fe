"""A latent cache's append against its definition in 64 bits."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_20507_amd import binding as B  # noqa: E402
from tests import latent_ref as L  # noqa: E402
from tests.gpu_util import device, say  # noqa: E402

pytestmark = pytest.mark.gpu

SIZES = [(128, 64, 512), (64, 32, 256), (128, 32, 256), (64, 64, 512)]  # nope, rope, rank


def make(dtype, R, H, size, far, seed=0):
    nope, rope, rank = size
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    q = torch.randn(R, H, nope + rope, generator=g, device="cuda")
    kv = 3.0 * torch.randn(R, rank + rope, generator=g, device="cuda")
    w = (1 + 0.2 * torch.randn(rank, generator=g, device="cuda")).to(dtype)
    P = (R + 15) // 16 + 2
    slot = torch.from_numpy(rng.permutation(P * 16)[:R].astype(np.int32)).to("cuda")
    pos = torch.from_numpy((far + rng.permutation(R)).astype(np.int32)).to("cuda")
    q_out = torch.full((R + 1, H, nope + rope), 9.0, dtype=dtype, device="cuda")
    pages = torch.full((P, 16, rank + rope), 5.0, dtype=dtype, device="cuda")
    return q, kv, w, P, slot, pos, q_out, pages


def call(dtype, R, H, size, theta, t):
    q, kv, w, P, slot, pos, q_out, pages = t
    B.spec_op_rope_latent(B.SPEC_F32 if dtype is torch.float32 else B.SPEC_BF16, R, H, *size, theta, 1e-5, q, kv, w, pos, slot,
                          P, q_out, pages)


def close(got, ref, dtype):
    """One rounding of each value, and fp32's: the norm's sum of 512 squares (in 8 chains and a tree, half of its
    error), root, quotient and products, under 16 steps of 2^-24; a rotation's two products and sum of
    values up to sqrt(2) times their pair's length."""
    pair = ref.abs().amax(-1, keepdim=True)
    tol = ref.abs() * (2.0 ** -8 if dtype is torch.bfloat16 else 0) + 16 * 2.0 ** -24 * (ref.abs() + pair)
    bad = ((got.double() - ref).abs() > tol).sum()
    assert int(bad) == 0, float((got.double() - ref).abs().max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R, H, size, far", [
    (1, 1, SIZES[0], 0), (1, 32, SIZES[0], 131071), (6, 32, SIZES[0], 2048), (5, 3, SIZES[1], 100), (17, 16, SIZES[2], 7),
    (381, 11, SIZES[3], 4096), (700, 32, SIZES[0], 0), (33, 65, SIZES[1], 1 << 30)])
def test_append(dtype, R, H, size, far):
    device()
    say("append", dtype, R, H, size, far)
    nope, rope, rank = size
    t = make(dtype, R, H, size, far, seed=R)
    q, kv, w, P, slot, pos, q_out, pages = t
    call(dtype, R, H, size, 5e5, t)
    rq, entry = L.append(q, kv, w, pos, H, *size, 5e5, 1e-5)
    close(q_out[:R, :, :nope], rq[..., :nope], dtype)
    close(q_out[:R, :, nope:], rq[..., nope:], dtype)
    assert (q_out[R:] == 9).all()
    flat = pages.view(-1, rank + rope)
    close(flat[slot.long(), :rank], entry[:, :rank], dtype)
    close(flat[slot.long(), rank:], entry[:, rank:], dtype)
    rest = torch.ones(P * 16, dtype=torch.bool, device="cuda")
    rest[slot.long()] = False
    assert (flat[rest] == 5).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_padding_rows_write_no_entry(dtype):
    device()
    size = SIZES[0]
    t = make(dtype, 9, 4, size, 50, seed=3)
    q, kv, w, P, slot, pos, q_out, pages = t
    slot[0], slot[4], slot[8] = -1, P * 16, -2147483648
    say("padding", dtype)
    call(dtype, 9, 4, size, 1e4, t)
    rq, entry = L.append(q, kv, w, pos, 4, *size, 1e4, 1e-5)
    close(q_out[:9, :, 128:], rq[..., 128:], dtype)
    flat = pages.view(-1, 576)
    kept = [1, 2, 3, 5, 6, 7]
    close(flat[slot[kept].long()], entry[kept], dtype)
    rest = torch.ones(P * 16, dtype=torch.bool, device="cuda")
    rest[slot[kept].long()] = False
    assert (flat[rest] == 5).all()


def test_values_that_are_not_finite_stay_in_their_row():
    device()
    say("append, not finite")
    t = make(torch.bfloat16, 4, 2, SIZES[1], 0, seed=4)
    q, kv, w, P, slot, pos, q_out, pages = t
    q[1, 0, 3], kv[2, 10], kv[3, 256 + 1] = math.nan, math.inf, math.nan
    call(torch.bfloat16, 4, 2, SIZES[1], 1e4, t)
    flat = pages.view(-1, 288)[slot.long()]
    assert torch.isnan(q_out[1, 0, 3]) and int(torch.isnan(q_out).sum()) == 1
    assert torch.isnan(flat[2, 10]) and (flat[2, :10] == 0).all() and torch.isfinite(flat[2, 256:]).all()
    assert torch.isnan(flat[3, 257]) and torch.isnan(flat[3, 257 + 16]) and int(torch.isnan(flat[3]).sum()) == 2
    assert torch.isfinite(flat[:2]).all()
