"""Comparisons of the latent cache's outputs (not collected: no test_ prefix)."""

import torch


def outside(got, ref, tol):
    """How many elements are not within tol of ref.  A NaN is within nothing."""
    return int((~((got.double() - ref).abs() <= tol)).sum())


def append_tol(ref, dtype):
    """One rounding of each value, and fp32's: the norm's sum of 512 squares (in 8 chains and a tree, half of its error), root,
    quotient and products, under 16 steps of 2^-24; a rotation's two products and sum of values up to sqrt(2) times their
    pair's length."""
    pair = ref.abs().amax(-1, keepdim=True)
    return ref.abs() * (2.0 ** -8 if dtype is torch.bfloat16 else 0) + 16 * 2.0 ** -24 * (ref.abs() + pair)
