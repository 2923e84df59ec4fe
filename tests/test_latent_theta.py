"""CPU check: a rotation base that is not finite is refused: theta^0 is 1, but the kernel's exp(-0 log theta) would be NaN."""

import os

import pytest

from paper_2607_20507_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="library not built")

P = 0x1000  # an address that no refused call may touch


def call(theta):  # (no rows: nothing is launched)
    return B.lib().spec_op_rope_latent(1, 0, 8, 128, 64, 512, theta, 1e-5, P, P, P, P, P, 10, P, P, None)


def test_an_infinite_theta():
    assert call(float("inf")) == B.SPEC_E_INVALID
    assert "spec_op_rope_latent" in B.lib().spec_last_error(None).decode()
    assert call(3.4e38) == B.SPEC_OK and call(1e-38) == B.SPEC_OK
