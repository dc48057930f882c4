"""Norms of gradients by block (frame, prediction row, output), beside the elementwise bounds of loss_reference.py: those grow with an utterance's length until a
part that is missing from a sum fits into them, a norm's share does not."""
import torch


def near(got, want, share, what):
    """Every block (all axes but the last) of `got` within `share` of the norm of `want`'s (and 2^-100: sums of numbers that fp32 does not hold count as zero)."""
    assert got.shape == want.shape, what
    got, want = got.double().to(want.device), want.double()
    off, size = (got - want).flatten(0, -2).norm(dim=1), want.flatten(0, -2).norm(dim=1)
    worst = float((off / size.clamp(min=2.0 ** -100)).max()) if off.numel() else 0.0
    assert bool((off <= share * size + 2.0 ** -100).all()), f"{what}: a block is off by {worst:.3g} of its norm"


# Of a block's norm.  bf16: the result is rounded to half a step, 2^-8 of it at most, and so is dx before its products (random rows of W and z do not cancel): 2^-7 in all,
# where every rounding is at its largest; z of the lattice in two planes and the counts' sums add less than 1e-3.  fp32: of paths of up to 500 arcs each is off by some
# 2^-20 (a logit of sums over 64, its norm), independently: 500^(1/2) 2^-20 = 2e-5, and sums over rows less.
SHARE = {"bf16": 1e-2, "f32": 1e-4}
