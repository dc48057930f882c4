"""Losses over the output layer where the bias masks outputs with finite values, as programs write masks: the same as outputs that are not there."""
import math

import pytest
import torch

from loss_reference import close, row_loss, transducer_loss
from test_gpu_losses import GRAD, api, check, lattice, rows

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


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("mask", (-1e4, -1e30, LOWEST))
@pytest.mark.parametrize("V1,first,end", [(300, 150, 300), (1025, 512, 1000), (70, 64, 70)])
def test_padded_outputs(V1, first, end, mask, dtype):
    """A vocabulary that is padded with masked outputs, whole blocks of columns of them; no row names one."""
    h, w, b, labels, weights = rows(140, 64, V1, dtype, V1)
    labels[(labels >= first) & (labels < end)] = 3
    masked, barred = b.clone(), b.clone()
    masked[first:end], barred[first:end] = mask, -math.inf
    ref = row_loss(h, w, barred, labels, weights=weights)
    check(api().label_loss(h, w, masked, labels, weights, grad=("h", "w", "b")), ref, "hwb")
    close(api().label_loss(h, w, masked, labels), *ref["loss"], "loss alone")
    at = torch.stack([labels, torch.where(labels >= 0, 5, -1).int()], 1)
    logits = torch.zeros(at.shape, device="cuda")
    check(api().distill_loss(h, w, masked, at, logits, 0.5, weights, grad=("h", "w", "b")), row_loss(h, w, barred, at, logits, 0.5, weights), "hwb")


@pytest.mark.parametrize("mask", (-1e4, -1e30, LOWEST))
def test_padded_outputs_of_a_lattice(mask):
    e, p, w, b, labels, frames, counts, weights = lattice(3, 20, 5, 32, 300, "bf16", 24)
    labels[labels >= 150] = 3
    masked, barred = b.clone(), b.clone()
    masked[150:299], barred[150:299] = mask, -math.inf
    check(api().transducer_loss(e, p, w, masked, labels, frames, counts, weights, grad=GRAD), transducer_loss(e, p, w, barred, labels, frames, counts, weights), GRAD)


@pytest.mark.parametrize("mask", (-1e4, -1e30, LOWEST))
def test_rows_that_name_a_masked_output(mask):
    """The loss is the mask's size; in the gradient the label takes all of its row's weight, as with an output that is barred."""
    h, w, b, labels, weights = rows(40, 64, 200, "f32", 25, left_out=0.0)
    labels[labels == 7] = 8
    labels[3] = 7
    masked, barred = b.clone(), b.clone()
    masked[7], barred[7] = mask, -math.inf
    ref = row_loss(h, w, barred, labels, weights=weights)
    loss, *grads = api().label_loss(h, w, masked, labels, weights, grad=("h", "w", "b"))
    assert torch.isfinite(loss).all() and abs(float(loss[3]) / -mask - 1) < 0.01
    for t, name in zip(grads, "hwb"):
        close(t, *ref[name], name)
