"""spec_token_logprobs on logits as far apart as fp32 holds them: their
differences pass the type's range, their differences over the temperature do not."""

import numpy as np
import pytest

from gpu_util import device, say
from test_gpu_logprobs import call, compare, reference

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BIG = float(np.finfo(np.float32).max)


@pytest.mark.parametrize("V", [7, 3000, 40000])
@pytest.mark.parametrize("temp", [1e30, 1e38, 3e38, np.inf])
def test_logits_of_both_ends_of_the_range(V, temp):
    dev = device()
    say("logprobs of far logits", V, temp)
    rng = np.random.default_rng(V)
    z = rng.choice(np.array([BIG, -BIG, 1e38, -2e38, 0, 1.5], np.float32), (5, V))
    z[1, 1:] = -BIG       # one at the top, all else at the bottom
    z[1, 0] = BIG
    z[2, : V // 2] = -np.inf
    z[3] = -BIG
    z[3, V - 1] = BIG
    z[:, V // 2] = BIG
    temps = np.full(5, temp, np.float32)
    tokens = np.array([V - 2, V - 1, V - 2, 0, V - 1], np.int32)
    n = min(6, V)
    # (float64 holds 1e300, at which finite logits are as equal and masked ones still masked)
    want = reference(z, np.minimum(temps.astype(np.float64), 1e300), tokens, n)
    got = call(torch.from_numpy(z).to(dev), torch.from_numpy(temps).to(dev), torch.from_numpy(tokens).to(dev), n, dev)
    compare(got, want, (V, temp))
