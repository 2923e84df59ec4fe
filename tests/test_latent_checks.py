"""CPU checks of the comparisons that the latent cache's GPU tests use: planted mistakes are counted."""

import math

import torch

from tests import latent_checks as K


def test_planted_values_are_counted():
    g = torch.Generator().manual_seed(0)
    ref = torch.randn(7, 3, 64, generator=g, dtype=torch.float64)
    for dtype in (torch.float32, torch.bfloat16):
        got, tol = ref.to(dtype), K.append_tol(ref, dtype)
        assert K.outside(got, ref, tol) == 0
        for i, x in enumerate([math.nan, math.inf, -math.inf, 9.0]):
            bad = got.clone()
            bad[i, 2, 60:62] = x
            assert K.outside(bad, ref, tol) == 2
        assert K.outside(torch.full_like(got, math.nan), ref, tol) == ref.numel()
        assert K.outside(got, ref + 0.01, tol) > 0  # the oracle off by a little
