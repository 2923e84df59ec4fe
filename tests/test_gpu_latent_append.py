"""A latent cache's append: every value of every row is written, and near its definition in 64 bits."""

import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2607_20507_amd import binding as B  # noqa: E402
from tests import latent_checks as K  # noqa: E402
from tests import latent_ref as L  # noqa: E402
from tests.gpu_util import device, say  # noqa: E402

pytestmark = pytest.mark.gpu


# nope, rope, rank; heads that one workgroup takes and that several share; one row to more than two a CU
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [(128, 64, 512), (64, 32, 256), (128, 32, 256), (64, 64, 512), (128, 64, 256), (64, 32, 512)])
@pytest.mark.parametrize("R, H, far", [(1, 1, 0), (6, 32, 131071), (17, 3, 1 << 30), (381, 11, 4096), (600, 33, 2048)])
def test_every_value_is_written_and_close(dtype, size, R, H, far):
    device()
    say("append", dtype, size, R, H, far)
    nope, rope, rank = size
    g = torch.Generator(device="cuda")
    g.manual_seed(R + H)
    rng = np.random.default_rng(R)
    q = torch.randn(R, H, nope + rope, generator=g, device="cuda")
    kv = 3.0 * torch.randn(R, rank + rope, generator=g, device="cuda")
    w = (1 + 0.2 * torch.randn(rank, generator=g, device="cuda")).to(dtype)
    P = (R + 15) // 16 + 2
    slot = torch.from_numpy(rng.permutation(P * 16)[:R].astype(np.int32)).to("cuda")
    pad = torch.zeros(R, dtype=torch.bool, device="cuda")
    if R > 16:
        pad[5::7] = True
        slot[pad] = -1
    pos = torch.from_numpy((far + rng.permutation(R)).astype(np.int32)).to("cuda")
    # NaN wherever nothing is written
    q_out = torch.full((R + 1, H, nope + rope), math.nan, dtype=dtype, device="cuda")
    pages = torch.full((P, 16, rank + rope), math.nan, dtype=dtype, device="cuda")
    B.spec_op_rope_latent(B.SPEC_F32 if dtype is torch.float32 else B.SPEC_BF16, R, H, nope, rope, rank, 5e5, 1e-5, q, kv, w, pos, slot,
                          P, q_out, pages)
    rq, entry = L.append(q, kv, w, pos, H, nope, rope, rank, 5e5, 1e-5)
    flat = pages.view(-1, rank + rope)
    held = flat[slot[~pad].long()]
    for got, ref in [(q_out[:R, :, :nope], rq[..., :nope]), (q_out[:R, :, nope:], rq[..., nope:]), (held[:, :rank], entry[~pad, :rank]),
                     (held[:, rank:], entry[~pad, rank:])]:
        assert torch.isfinite(got).all()
        assert K.outside(got, ref, K.append_tol(ref, dtype)) == 0
    assert torch.isnan(q_out[R:]).all()
    rest = torch.ones(P * 16, dtype=torch.bool, device="cuda")
    rest[slot[~pad].long()] = False
    assert torch.isnan(flat[rest]).all()
