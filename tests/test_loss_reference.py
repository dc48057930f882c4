"""The plain references of the losses: against torch's autograd in 64 bits, and against differences."""
import math

import pytest
import torch

from loss_reference import row_loss, transducer_loss


def random_lattice(seed, B=3, T=5, U=3, H=4, V1=6):
    g = torch.Generator().manual_seed(seed)
    e, p = torch.randn((B, T, H), generator=g, dtype=torch.float64), torch.randn((B, U + 1, H), generator=g, dtype=torch.float64)
    w, b = torch.randn((V1, H), generator=g, dtype=torch.float64), torch.randn(V1, generator=g, dtype=torch.float64)
    labels = torch.randint(0, V1 - 1, (B, U), generator=g, dtype=torch.int32)
    return e, p, w, b, labels, torch.tensor([T, 2, 0][:B]), torch.tensor([U, 0, 1][:B]), torch.rand(B, generator=g)


def all_paths(lp, y):
    """-log of the sum over every sequence of blanks and labels, by recursion over paths."""
    T = lp.shape[0]

    def walk(t, u):
        if t == T:
            return [torch.zeros((), dtype=lp.dtype)] if u == len(y) else []
        found = [lp[t, u, -1] + rest for rest in walk(t + 1, u)]
        if u < len(y):
            found += [lp[t, u, int(y[u])] + rest for rest in walk(t, u + 1)]
        return found
    return -torch.logsumexp(torch.stack(walk(0, 0)), 0)


@pytest.mark.parametrize("seed", range(3))
def test_transducer_reference_is_the_sum_over_paths(seed):
    e, p, w, b, labels, frames, counts, weights = random_lattice(seed)
    leaves = [t.clone().requires_grad_() for t in (e, p, w, b)]
    total = 0.0
    want = []
    for i in range(3):
        T, U = int(frames[i]), int(counts[i])
        if T == 0:
            want.append(torch.zeros((), dtype=torch.float64))
            continue
        z = torch.relu(leaves[0][i, :T, None] + leaves[1][i, None, :U + 1])
        lp = torch.log_softmax(z @ leaves[2].t() + leaves[3], 2)
        want.append(all_paths(lp, labels[i, :U]))
        total = total + weights[i].double() * want[-1]
    total.backward()
    ref = transducer_loss(e, p, w, b, labels, frames, counts, weights)
    assert torch.allclose(ref["loss"][0], torch.stack(want).detach(), rtol=1e-12)
    for name, leaf in zip("epwb", leaves):
        assert torch.allclose(ref[name][0], leaf.grad, rtol=1e-10, atol=1e-12), name


@pytest.mark.parametrize("tau", (1.0, 2.5))
def test_row_reference_against_autograd(tau):
    g = torch.Generator().manual_seed(5)
    h, w, b = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((7, 4), (9, 4), (9,)))
    weights = torch.rand(7, generator=g)
    labels = torch.randint(0, 9, (7, 3), generator=g, dtype=torch.int32)
    labels[2] = -1
    labels[3, 1] = -1
    labels[4, 0] = labels[4, 2]
    logits = torch.randn((7, 3), generator=g)
    logits[5, 1] = -math.inf
    leaves = [t.clone().requires_grad_() for t in (h, w, b)]
    x = torch.log_softmax((leaves[0] @ leaves[1].t() + leaves[2]) / tau, 1)
    losses = []
    for n in range(7):
        ks = [k for k in range(3) if labels[n, k] >= 0 and logits[n, k] > -math.inf]
        if not ks:
            losses.append(torch.zeros((), dtype=torch.float64))
            continue
        q = torch.softmax(logits[n, ks].double() / tau, 0)
        losses.append(tau * tau * sum(q[j] * (q[j].log() - x[n, int(labels[n, k])]) for j, k in enumerate(ks)))
    (torch.stack(losses) * weights.double()).sum().backward()
    ref = row_loss(h, w, b, labels, logits, tau, weights)
    assert torch.allclose(ref["loss"][0], torch.stack(losses).detach(), rtol=1e-12)
    for name, leaf in zip("hwb", leaves):
        assert torch.allclose(ref[name][0], leaf.grad, rtol=1e-10, atol=1e-12), name
    plain = row_loss(h, w, b, labels[:, 0].contiguous())
    x = torch.log_softmax(h @ w.t() + b, 1)
    for n in range(7):
        want = -float(x[n, int(labels[n, 0])]) if labels[n, 0] >= 0 else 0.0
        assert abs(float(plain["loss"][0][n]) - want) < 1e-12


def test_row_reference_against_differences():
    g = torch.Generator().manual_seed(6)
    h, w, b = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((4, 3), (5, 3), (5,)))
    labels = torch.tensor([0, 4, -1, 2], dtype=torch.int32)
    ref = row_loss(h, w, b, labels)
    step = torch.randn(w.shape, generator=g, dtype=torch.float64)
    at = lambda s: float(row_loss(h, w + s * step, b, labels)["loss"][0].sum())  # noqa: E731
    assert abs((at(1e-5) - at(-1e-5)) / 2e-5 - float((ref["w"][0] * step).sum())) < 1e-8
