"""Losses over the output layer of more rows than a workspace holds at a time.  That a call takes several pieces is asserted from its workspace, which does
not grow with the rows any more."""
import ctypes as C

import pytest
import torch

from loss_norms import SHARE, near
from loss_reference import close, row_loss, transducer_loss
from test_gpu_losses import GRAD, api, check, lattice, rows

pytestmark = pytest.mark.gpu


def query(name, w, *sizes):
    from paper_2505_13765_amd.binding import WIND_BF16, WIND_F32, OutputLayer, load_library

    lay, n = OutputLayer(w.data_ptr(), None, w.shape[1], *w.shape, WIND_BF16 if w.dtype == torch.bfloat16 else WIND_F32), C.c_size_t(0)
    assert getattr(load_library(), name)(C.byref(lay), *sizes, C.byref(n)) == 0
    return n.value


def rows_in_pieces(w, N, K, grads):
    """Whether a sixteenth of the rows adds less than a tenth of its panels' bytes: the workspace held no more rows before."""
    V1, H = w.shape
    sizes = [query("wind_row_loss_workspace_bytes", w, n, K, grads) for n in (N * 15 // 16, N)]
    return sizes[1] - sizes[0] < N // 16 * (2 if w.dtype == torch.bfloat16 else 6) * (H + (V1 if grads else 0)) / 10


def nodes_in_pieces(w, B, T, U, grads):
    V1, H = w.shape
    sizes = [query("wind_transducer_loss_workspace_bytes", w, B, t, U, grads) for t in (T * 15 // 16, T)]
    z, dx = (4, 2) if w.dtype == torch.bfloat16 else (6, 6)
    return sizes[1] - sizes[0] < B * (T // 16) * (U + 1) * (z * H + (dx * V1 + 4 * H if grads else 0)) / 10


def row_reference(h, w, b, labels, logits=None, tau=1.0, weights=None, step=3000):
    """row_loss, piece by piece: its fp64 logits of all rows would not fit."""
    part = lambda t, i: None if t is None else t[i:i + step]  # noqa: E731
    refs = [row_loss(part(h, i), w, b, part(labels, i), part(logits, i), tau, part(weights, i)) for i in range(0, len(h), step)]
    out = {k: tuple(torch.cat([r[k][x] for r in refs]) for x in range(2)) for k in ("loss", "h")}
    for k in ("w", "b"):
        value = sum(r[k][0] for r in refs)
        out[k] = value, sum(r[k][1] for r in refs) + 2.0 ** -24 * len(refs) * value.abs()   # (added up once more per piece)
    return out


def check_norms(got, ref, names, share):
    for t, name in zip(got[1:], names):
        want = ref[name][0]
        near(t.double().reshape(1, -1), want.reshape(1, -1), share, name)
        if name in "ehp":
            near(t, want, share, name + " by block")


@pytest.mark.parametrize("dtype,N,H,V1", [("bf16", 24001, 64, 65537), ("f32", 16001, 96, 30001)])
def test_label_loss_in_pieces(dtype, N, H, V1):
    """A last piece of few rows, and pieces without any row that counts."""
    h, w, b, labels, weights = rows(N, H, V1, dtype, 31, left_out=0.0)
    assert rows_in_pieces(w, N, 1, 1)
    for end in (N, N // 3, 0):
        labels[end:] = -1
        ref = row_reference(h, w, b, labels, weights=weights)
        got = api().label_loss(h, w, b, labels, weights, grad=("h", "w", "b"))
        check(got, ref, "hwb")
        check_norms(got, ref, "hwb", SHARE[dtype])


@pytest.mark.parametrize("dtype,N,H,V1,K", [("bf16", 14001, 48, 65537, 4), ("bf16", 30001, 64, 30001, 16), ("f32", 12001, 64, 20001, 6)])
def test_distill_loss_in_pieces(dtype, N, H, V1, K):
    """Sorted entries of a later piece among them."""
    h, w, b, _, weights = rows(N, H, V1, dtype, 32, left_out=0.0)
    assert rows_in_pieces(w, N, K, 1)
    g = torch.Generator().manual_seed(33)
    labels = torch.randint(-1, V1, (N, K), generator=g, dtype=torch.int32)
    labels[::3, 1] = labels[::3, 0]
    logits = 2 * torch.randn((N, K), generator=g)
    labels, logits = labels.cuda(), logits.cuda()
    ref = row_reference(h, w, b, labels, logits, 2.0, weights)
    got = api().distill_loss(h, w, b, labels, logits, 2.0, weights, grad=("h", "w", "b"))
    check(got, ref, "hwb")
    check_norms(got, ref, "hwb", SHARE[dtype])


@pytest.mark.parametrize("grad", (None, ("h", "w", "b")))
def test_few_wide_rows_in_pieces(grad):
    """Few rows, few outputs and hidden rows so long that a piece holds part of them: each piece's column blocks are joined by the launch that makes them."""
    N, H, V1 = 4096, 80000, 300
    h, w, b, labels, weights = rows(N, H, V1, "f32", 34, left_out=0.0)
    assert rows_in_pieces(w, N, 1, 0 if grad is None else 1)
    ref = row_loss(h, w, b, labels, weights=weights)
    got = api().label_loss(h, w, b, labels, weights, grad=grad)
    if grad is None:
        close(got, *ref["loss"], "loss")
        return
    check(got, ref, grad)
    check_norms(got, ref, grad, SHARE["f32"])


@pytest.mark.parametrize("grad", (None, GRAD))
def test_few_wide_nodes_in_pieces(grad):
    B, T, U, H = 2, 100, 9, 110000
    a = lattice(B, T, U, H, 12, "f32", 35)
    a[0], a[1], a[4] = torch.nan_to_num(a[0]), torch.nan_to_num(a[1], posinf=0.0), a[4].clamp(min=0)
    a[5][:], a[6][:] = T, U
    assert nodes_in_pieces(a[2], B, T, U, 0 if grad is None else 1)
    ref = transducer_loss(*a)
    got = api().transducer_loss(*a, grad=grad)
    if grad is None:
        close(got, *ref["loss"], "loss")
        return
    check(got, ref, GRAD)
    check_norms(got, ref, GRAD, SHARE["f32"])


@pytest.mark.parametrize("dtype,N,H,V1", [("bf16", 40001, 640, 65537), ("bf16", 900001, 48, 4097), ("f32", 20000, 320, 65537)])
def test_scores_of_many_rows(dtype, N, H, V1):
    """Losses alone, of rows that a step takes too: the same bits as its losses, and the first and last rows' against the reference."""
    h, w, b, labels, weights = rows(N, H, V1, dtype, 37)
    loss = api().label_loss(h, w, b, labels)
    assert torch.equal(loss, api().label_loss(h, w, b, labels, weights, grad=("b",))[0])
    for part in (slice(0, 500), slice(N - 500, N)):
        close(loss[part], *row_loss(h[part], w, b, labels[part])["loss"], "loss")
    assert not loss[labels < 0].any() and (loss[labels >= 0] > 0).all()


@pytest.mark.parametrize("dtype,B,T,U,H,V1", [("bf16", 16, 750, 120, 640, 8193), ("bf16", 32, 750, 120, 48, 4097), ("f32", 8, 250, 40, 96, 8193)])
def test_scores_of_many_nodes(dtype, B, T, U, H, V1):
    a = lattice(B, T, U, H, V1, dtype, 38)
    loss = api().transducer_loss(*a)
    assert torch.equal(loss, api().transducer_loss(*a, grad=("b",))[0]) and torch.isfinite(loss).all()
    for i in (0, B - 1):
        one = [t[i:i + 1] for t in a[:2]] + a[2:4] + [t[i:i + 1] for t in a[4:]]
        close(loss[i:i + 1], *transducer_loss(*one)["loss"], "loss")


@pytest.mark.parametrize("dtype,B,T,U,H,V1", [("bf16", 24, 400, 60, 64, 2049), ("f32", 8, 250, 40, 32, 4097), ("bf16", 3, 2000, 60, 65, 3001)])
def test_lattices_in_pieces(dtype, B, T, U, H, V1):
    """Frames and labels whose sums go over a piece's end, utterances that end early or do not count, pieces without nodes; with dz read once and apart."""
    a = lattice(B, T, U, H, V1, dtype, 36)
    a[0], a[1], a[4] = torch.nan_to_num(a[0]), torch.nan_to_num(a[1], posinf=0.0), a[4].clamp(min=0)
    a[5][:], a[6][:] = T, U
    assert nodes_in_pieces(a[2], B, T, U, 1)
    a[5][1], a[6][2] = T // 2 + 3, U // 3
    for shorter in (False, True):
        if shorter:
            a[5][1:] = 0
            a[5][0] = T // 3
        ref = transducer_loss(*a)
        got = api().transducer_loss(*a, grad=GRAD)
        check(got, ref, GRAD)
        check_norms(got, ref, GRAD, SHARE[dtype])
        for part in (("e",), ("p",)):       # (the folds apart)
            some = api().transducer_loss(*a, grad=part)
            check_norms(some, ref, part, SHARE[dtype])


def test_a_large_lattice_in_one_piece():
    """dz read once for both of its folds: shares of the norms, frame by frame and prediction row by prediction row."""
    a = lattice(3, 203, 40, 701, 40, "bf16", 16)
    a[0], a[1], a[4] = torch.nan_to_num(a[0]), torch.nan_to_num(a[1], posinf=0.0), a[4].clamp(min=0)
    a[5][1] = 0
    check_norms(api().transducer_loss(*a, grad=GRAD), transducer_loss(*a), GRAD, SHARE["bf16"])


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_one_workspace_for_all_calls(dtype):
    """A buffer for the largest call, with whatever the last one left in it, serves smaller ones and scores: the same bits as with one of the call's own size."""
    from paper_2505_13765_amd.binding import WIND_BF16, WIND_F32, OutputLayer, load_library

    lib, most, H, V1 = load_library(), 12000, 200, 5000
    h, w, b, labels, weights = rows(most, H, V1, dtype, 39)
    lay = OutputLayer(w.data_ptr(), b.data_ptr(), H, V1, H, WIND_BF16 if dtype == "bf16" else WIND_F32)
    size = query("wind_row_loss_workspace_bytes", w, most, 1, 1)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    for N in (12000, 11000, 3000, 257, 128, 1, 9999):
        for grad in (("h", "w", "b"), None):
            want = api().label_loss(h[:N], w, b, labels[:N], weights[:N], grad=grad)
            outs = [torch.full_like(t, 7.0) for t in (want if grad else (want,))]
            ptrs = [t.data_ptr() for t in outs] + [None] * (4 - len(outs))
            assert lib.wind_label_loss(C.byref(lay), h.data_ptr(), H, labels.data_ptr(), weights.data_ptr(), N, *ptrs, ws.data_ptr(), size,
                                       torch.cuda.current_stream().cuda_stream) == 0
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(outs, want if grad else (want,))), (N, grad)
    size = query("wind_transducer_loss_workspace_bytes", w, 6, 60, 20, 1)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    for B, T, U in ((6, 60, 20), (5, 60, 19), (6, 10, 20), (1, 1, 0), (6, 59, 20)):
        e, p, _, _, y, frames, counts, weights = lattice(B, T, U, H, V1, dtype, 40 + T)
        want = api().transducer_loss(e, p, w, b, y, frames, counts, weights, grad=GRAD)
        outs = [torch.full_like(t, 7.0) for t in want]
        assert lib.wind_transducer_loss(C.byref(lay), e.data_ptr(), e.stride(0), e.stride(1), p.data_ptr(), p.stride(0), p.stride(1), y.data_ptr(), frames.data_ptr(),
                                        counts.data_ptr(), weights.data_ptr(), B, T, U, *(t.data_ptr() for t in outs), ws.data_ptr(), size,
                                        torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want)), (B, T, U)
