"""Losses over the output layer where the bias masks outputs with finite values, as programs write masks: the same as outputs that are not there."""
import math

import pytest
import torch

from loss_reference import close, transducer_loss
from test_gpu_losses import GRAD, api, check, lattice

pytestmark = pytest.mark.gpu

LOWEST = torch.finfo(torch.float32).min


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("mask", (-1e9, -2e9, -1e10, -1e30, LOWEST))
def test_transcripts_that_name_a_masked_output(mask, dtype):
    """A path through an arc of probability e^mask has none: loss +inf, no gradient, and the other utterances are as with an output that is barred."""
    e, p, w, b, labels, frames, counts, weights = lattice(4, 20, 5, 32, 20, dtype, 21)
    e, p, labels = torch.nan_to_num(e), torch.nan_to_num(p, posinf=0.0), labels.clamp(min=0)
    frames[:], counts[:] = 20, 5
    labels[labels == 4] = 5
    labels[0, 2], labels[2, 4] = 4, 4
    masked, barred = b.clone(), b.clone()
    masked[4], barred[4] = mask, -math.inf
    ref = transducer_loss(e, p, w, barred, labels, frames, counts, weights)
    got = api().transducer_loss(e, p, w, masked, labels, frames, counts, weights, grad=GRAD)
    assert got[0][0] == math.inf and got[0][2] == math.inf
    check(got, ref, GRAD)
    close(api().transducer_loss(e, p, w, masked, labels, frames, counts, weights), *ref["loss"], "loss alone")


@pytest.mark.parametrize("mask", (-1e9, -2e9, -1e10, -1e30, LOWEST))
def test_blank_is_masked(mask):
    """No path ends: every loss is +inf and every gradient zero."""
    e, p, w, b, labels, frames, counts, weights = lattice(3, 20, 5, 32, 20, "f32", 22)
    b[-1] = mask
    e, p = torch.nan_to_num(e), torch.nan_to_num(p, posinf=0.0)
    loss, *grads = api().transducer_loss(e, p, w, b, labels, frames, counts, weights, grad=GRAD)
    assert torch.equal(loss, torch.full_like(loss, math.inf))
    for t in grads:
        assert not t.any()


@pytest.mark.parametrize("mask", (-1e4, -1e7))
def test_improbable_arcs_keep_their_size(mask):
    """Probabilities far below those that fp32 holds, on one arc; the losses are of the mask's size, known to fp32's rounding of the logit (and 2^-20 beside)."""
    e, p, w, b, labels, frames, counts, weights = lattice(2, 20, 5, 32, 20, "f32", 23)
    e, p, labels = torch.nan_to_num(e), torch.nan_to_num(p, posinf=0.0), labels.clamp(min=0)
    counts[:] = 5
    labels[labels == 4] = 5
    labels[:, 1] = 4
    b[4] = mask
    loss, ref = api().transducer_loss(e, p, w, b, labels, frames, counts), transducer_loss(e, p, w, b, labels, frames, counts)["loss"][0]
    assert float(ref.min()) > -0.9 * mask
    assert ((loss.double().cpu() - ref).abs() <= 2.0 ** -20 * ref).all()
