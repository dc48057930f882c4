"""How exact the losses' gradients are where few rows count among many, and against differences along the gradient itself."""
import pytest
import torch

from loss_reference import transducer_loss
from test_gpu_losses import GRAD, api, lattice

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,count,V1", [(200, 5, 400), (256, 128, 400), (5000, 60, 400), (20001, 128, 3001), (700, 1, 90)])
def test_few_rows_that_count_among_many(N, count, V1):
    """Padding does not cost precision: gradients of up to 128 rows that count are off by the result's own rounding and what dx on 16 bits leaves, as in
    test_gradients_of_few_rows_are_only_rounded_once, whose bound this is (the weight 1 + 2^-8 lies between two bf16 values)."""
    H = 64
    g = torch.Generator().manual_seed(N)
    h, w = (0.25 * torch.randn(s, H, generator=g) for s in (N, V1))
    b, labels = 0.1 * torch.randn(V1, generator=g), torch.full((N,), -1, dtype=torch.int32)
    at = torch.randperm(N, generator=g)[:count].sort()[0]
    labels[at] = torch.randint(0, V1, (count,), generator=g, dtype=torch.int32)
    h, w, c = h.bfloat16(), w.bfloat16(), 1 + 2.0**-8
    _, dh, dw = api().label_loss(h.cuda(), w.cuda(), b.cuda(), labels.cuda(), weights=torch.full((N,), c).cuda(), grad=("h", "w"))
    assert int(dh.any(dim=1).sum()) == count
    dh, h, w, b, labels = dh[at.cuda()], h[at].double(), w.double(), b.double(), labels[at]
    p = torch.softmax(h @ w.T + b, dim=1)
    dx = c * (p - torch.nn.functional.one_hot(labels.long(), V1))
    logit = 2 * (H + 2) * 2.0**-24 * (h.abs() @ w.abs().T + b.abs()).amax(1, keepdim=True) + 2.0**-20
    off = 2.0**-16 * dx.abs() + c * p * logit
    for got, ref, bound in ((dh, dx @ w, off @ w.abs() + (V1 + 8) * 2.0**-24 * (dx.abs() @ w.abs())),
                            (dw, dx.T @ h, off.T @ h.abs() + (count + 8) * 2.0**-24 * (dx.abs().T @ h.abs()))):
        err = (got.double().cpu() - ref).abs()
        assert (err <= 2.0**-8 * (ref.abs() + bound) + bound + 2.0**-133).all(), (err - 2.0**-8 * ref.abs()).max()


def test_gradients_against_differences_along_them():
    """Along the reference's gradient of each input, normalised, so that the slope is that gradient's norm; fp32.  A central difference over 2 s is off by the losses' own
    bounds over s and by its truncation, which is that of the same difference of the reference: a small share of the slope."""
    s = 2.0 ** -5
    a = lattice(2, 8, 4, 24, 20, "f32", 10)
    for i in (0, 1):
        a[i] = torch.nan_to_num(a[i], posinf=0.0)
    got, ref = api().transducer_loss(*a, grad=GRAD), transducer_loss(*a)
    weights = a[7].double().cpu()
    for k, i in zip(GRAD, range(4)):
        step = (ref[k][0] / ref[k][0].norm()).float()
        step = (step / step.double().norm()).float().cuda()
        mine, exact, bound = [], [], 0.0
        for sign in (1, -1):
            moved = list(a)
            moved[i] = a[i] + sign * s * step
            there = transducer_loss(*moved)["loss"]
            mine.append(float((api().transducer_loss(*moved).double().cpu() * weights).sum()))
            exact.append(float((there[0] * weights).sum()))
            bound += float((there[1] * weights).sum()) / (2 * s)
        along = lambda x: float((x.double() * step.double()).sum())  # noqa: E731
        slope = along(ref[k][0])
        bound += abs((exact[0] - exact[1]) / (2 * s) - slope)
        assert bound < 0.02 * slope, (k, bound, slope)
        assert abs((mine[0] - mine[1]) / (2 * s) - slope) <= bound, (k, mine, bound)
        assert abs(along(got[1 + GRAD.index(k)]) - slope) <= 1e-4 * slope, (k, slope)


@pytest.mark.parametrize("N,first", [(1000, 0), (5000, 40)])
def test_a_weight_that_all_rows_share_is_not_rounded(N, first):
    """bf16 gradients of many rows of the weight c = 1 + 2^-8, which lies between two bf16 values, behind `first` rows of weight zero.  dx / c is p_v to bf16, off by 2^-8 of it
    at most, and p - 1 at the label, off by p or half a step below one, 2^-9, whichever is less; c itself is multiplied in fp32.  Times c before its rounding, every
    row's label would be off by almost 2^-8.  Beside that, logits, products and the result's rounding as in test_few_rows_that_count_among_many."""
    H, V1, c = 64, 4000, 1 + 2.0**-8
    g = torch.Generator().manual_seed(N)
    h, w = (0.25 * torch.randn(s, H, generator=g) for s in (N, V1))
    b, labels, weights = 0.1 * torch.randn(V1, generator=g), torch.randint(0, V1, (N,), generator=g, dtype=torch.int32), torch.full((N,), c)
    weights[:first] = 0
    h, w = h.bfloat16(), w.bfloat16()
    _, dh, dw, db = api().label_loss(h.cuda(), w.cuda(), b.cuda(), labels.cuda(), weights=weights.cuda(), grad=("h", "w", "b"))
    h, w, b = h.double(), w.double(), b.double()
    p, one = torch.softmax(h @ w.T + b, dim=1), torch.nn.functional.one_hot(labels.long(), V1).double()
    weights = weights.double()[:, None]
    dx = weights * (p - one)
    logit = 2 * (H + 2) * 2.0**-24 * (h.abs() @ w.abs().T + b.abs()).amax(1, keepdim=True) + 2.0**-20
    exact = weights * p * logit + 2.0**-22 * dx.abs()
    off = exact + weights * torch.where(one > 0, p.clamp(max=2.0**-9), 2.0**-8 * p)
    for got, ref, bound in ((dh, dx @ w, off @ w.abs() + (V1 + 8) * 2.0**-24 * (dx.abs() @ w.abs())),
                            (dw, dx.T @ h, off.T @ h.abs() + (N + 8) * 2.0**-24 * (dx.abs().T @ h.abs()))):
        err = (got.double().cpu() - ref).abs()
        assert (err <= 2.0**-8 * (ref.abs() + bound) + bound + 2.0**-133).all(), (err - 2.0**-8 * ref.abs()).max()
    assert ((db.double().cpu() - dx.sum(0)).abs() <= exact.sum(0) + (N + 40) * 2.0**-24 * dx.abs().sum(0)).all()
