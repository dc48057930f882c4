"""That the share of a block's norm which loss_norms allows tells a missing or doubled part of a sum from roundings: mistakes planted in the reference's sums."""
import math

import pytest
import torch

from loss_norms import SHARE, near
from loss_reference import transducer_loss


def parts(T=203, U=40, H=32, V1=20, seed=1):
    """Inputs of one utterance and the gradient of its nodes' hidden rows [T, U + 1, H], by autograd through the lattice, diagonal by diagonal."""
    g = torch.Generator().manual_seed(seed)
    e, p, w = (torch.randn(s, H, generator=g, dtype=torch.float64) for s in (T, U + 1, V1))
    w, b, y = w / math.sqrt(H), torch.randn(V1, generator=g, dtype=torch.float64), torch.randint(0, V1 - 1, (U,), generator=g)
    z = (e[:, None] + p[None]).clamp(min=0).requires_grad_()
    lp = torch.log_softmax(z @ w.T + b, 2)
    blank, emit = lp[:, :, -1], lp[:, torch.arange(U), y]
    run = torch.cat([emit.new_zeros(T, 1), emit.cumsum(1)], 1)      # labels emitted on one frame before u
    alpha = run[0]
    for t in range(1, T):
        alpha = run[t] + torch.logcumsumexp(alpha + blank[t - 1] - run[t], 0)
    (-(alpha[U] + blank[T - 1, U])).backward()
    dz = torch.where(z > 0, z.grad, 0.0)
    return (e[None], p[None], w, b, y[None].int(), torch.tensor([T]), torch.tensor([U])), dz.detach()


@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_missing_parts_show(dtype):
    inputs, dz = parts()
    share = SHARE["bf16" if dtype is torch.bfloat16 else "f32"]
    ref = transducer_loss(*inputs)
    rounded = lambda t: t.to(dtype).double()  # noqa: E731
    near(rounded(dz.sum(1))[None], ref["e"][0], share, "e")           # what is right passes
    near(rounded(dz.sum(0))[None], ref["p"][0], share, "p")
    planted = {}
    for f in (0, 96, 200):
        lost = dz.clone()
        lost[f:f + 8] = 0                                             # eight frames of a prediction row's sum
        planted[f"part {f}"] = lost
    flat = dz.reshape(-1, dz.shape[2])
    for first, times in ((4096, 0.0), (4096, 2.0), (8000, 0.0)):     # rows behind a chunk's end: lost, or added twice
        lost = flat.clone()
        lost[first:] *= times
        planted[f"rows from {first} times {times}"] = lost.view_as(dz)
    for u in range(0, dz.shape[1], 13):                               # one in 41 of a frame's rows
        lost = dz.clone()
        lost[:, u] = 0
        planted[f"label {u}"] = lost
    for what, wrong in planted.items():
        caught = 0
        for name, got in (("e", wrong.sum(1)), ("p", wrong.sum(0))):
            try:
                near(rounded(got)[None], ref[name][0], share, name)
            except AssertionError:
                caught += 1
        assert caught, what
