"""SpecSession.token_logprobs: its checks of arguments, other default types,
another stream."""

import numpy as np
import pytest

from test_gpu_fork import models, session
from workloads import uniform_prompts

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def verified():
    cfg, pair = models("fp32")
    s = session(pair, draft=False)
    s.prefill([1, 2], uniform_prompts(cfg.seed + 31, [20, 35], cfg.target.vocab))
    s.target_forward([1, 2])
    yield s
    s.close()


def test_lists_of_another_length_are_refused(verified):
    for bad in ([3], [3, 4, 5], []):
        with pytest.raises(ValueError):
            verified.token_logprobs(tokens=bad)
        with pytest.raises(ValueError):
            verified.token_logprobs(temps=[0.5] * len(bad))
    lp, h, ids, top = verified.token_logprobs(tokens=[3, 4], temps=[0.5, 1.0], n_top=2)
    z = verified.last_logits().double().cpu()
    want = torch.log_softmax(z / torch.tensor([[0.5], [1.0]], dtype=torch.float64), -1)
    assert np.allclose(lp.cpu(), want[[0, 1], [3, 4]], atol=1e-4) and np.allclose(top.cpu(), torch.topk(want, 2)[0], atol=1e-4)


def test_with_another_default_type_and_stream(verified):
    want = verified.token_logprobs(tokens=[3, 4], n_top=3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.set_default_dtype(torch.float64)
    try:
        got = verified.token_logprobs(tokens=[3, 4], n_top=3)
        other = verified.token_logprobs(tokens=[3, 4], n_top=3, stream=side)
    finally:
        torch.set_default_dtype(torch.float32)
    torch.cuda.synchronize()
    for w, g, o in zip(want, got, other):
        assert torch.equal(w, g) and torch.equal(w, o)
