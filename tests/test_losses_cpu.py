"""Losses over the output layer, without a GPU: refusals of the C entry points and of the Python functions, workspace sizes."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    from paper_2505_13765_amd import binding, build

    if build.stale():
        build.build(True)
    return binding.load_library()


def layer(V1=33, H=64, dtype=0, w=4096, b=0, stride=None):
    from paper_2505_13765_amd.binding import OutputLayer

    return OutputLayer(w, b, H if stride is None else stride, V1, H, dtype)


def rows_size(lib, lay, N, K=1, grads=1):
    n = C.c_size_t(0)
    return lib.wind_row_loss_workspace_bytes(C.byref(lay), N, K, grads, C.byref(n)), n.value


def lattice_size(lib, lay, B, T, U, grads=1):
    n = C.c_size_t(0)
    return lib.wind_transducer_loss_workspace_bytes(C.byref(lay), B, T, U, grads, C.byref(n)), n.value


@pytest.mark.parametrize("bad", [dict(V1=1), dict(H=0, stride=1), dict(dtype=2), dict(stride=63), dict(w=4097), dict(b=2), dict(w=0)])
def test_bad_layers_are_refused(lib, bad):
    from paper_2505_13765_amd.binding import WIND_ERR_ARG

    assert rows_size(lib, layer(**bad), 8)[0] == WIND_ERR_ARG
    assert lattice_size(lib, layer(**bad), 1, 4, 2)[0] == WIND_ERR_ARG


def test_sizes_out_of_range_are_refused(lib):
    from paper_2505_13765_amd.binding import WIND_ERR_ARG, WIND_ERR_UNSUPPORTED, WIND_OK

    assert rows_size(lib, layer(), -1)[0] == WIND_ERR_ARG
    assert rows_size(lib, layer(), 1 << 31)[0] == WIND_ERR_ARG
    assert rows_size(lib, layer(), 8, K=0)[0] == WIND_ERR_ARG
    assert rows_size(lib, layer(), 8, K=1025)[0] == WIND_ERR_UNSUPPORTED
    assert rows_size(lib, layer(V1=1 << 20, H=2048), 8)[0] == WIND_ERR_UNSUPPORTED
    assert lattice_size(lib, layer(), 0, 4, 2)[0] == WIND_ERR_ARG
    assert lattice_size(lib, layer(), 1, -1, 2)[0] == WIND_ERR_ARG
    assert lattice_size(lib, layer(), 1, 4, 4096)[0] == WIND_ERR_UNSUPPORTED
    assert lattice_size(lib, layer(), 1 << 10, 1 << 11, 1 << 10)[0] == WIND_ERR_UNSUPPORTED
    for ok in (rows_size(lib, layer(), 0), rows_size(lib, layer(V1=2, H=1, stride=1), 1, K=1024), lattice_size(lib, layer(), 1, 0, 0)):
        assert ok[0] == WIND_OK and ok[1] > 0


def test_workspace_is_bounded_by_the_chunk(lib):
    """A million rows of 65537 outputs have 131 GB of bf16 logits; the workspace holds a piece of them."""
    small, large = rows_size(lib, layer(V1=65537, H=64, dtype=1), 1 << 16)[1], rows_size(lib, layer(V1=65537, H=64, dtype=1), 1 << 20)[1]
    assert large < 2 << 30 and large - small < 64 << 20
    assert lattice_size(lib, layer(V1=8193, H=640, dtype=1), 64, 1000, 100)[1] < 2 << 30


def test_entry_points_check_before_they_launch(lib):
    """Pointers here are made up: a call that touched them would not return an argument error."""
    from paper_2505_13765_amd.binding import WIND_ERR_ARG

    lay, p = layer(), 4096
    need = rows_size(lib, lay, 8)[1]

    def label(lay=lay, h=p, stride=64, labels=p, N=8, loss=p, dh=p, ws=p, size=need):
        return lib.wind_label_loss(C.byref(lay) if lay else None, h, stride, labels, None, N, loss, dh, None, None, ws, size, None)

    for bad in (dict(lay=None), dict(h=None), dict(h=p + 1), dict(stride=63), dict(labels=None), dict(N=-1), dict(N=1 << 31), dict(loss=None), dict(dh=p + 2),
                dict(ws=None), dict(ws=p + 128), dict(size=need // 2)):
        assert label(**bad) == WIND_ERR_ARG, bad
    assert label(size=1) == WIND_ERR_ARG and b"needs" in lib.wind_last_error()

    def distill(logits=p, K=2, tau=1.0):
        return lib.wind_distill_loss(C.byref(lay), p, 64, p, logits, K, tau, None, 8, p, None, None, None, p, 1 << 40, None)

    for bad in (dict(logits=None), dict(K=0), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("inf")), dict(tau=float("nan")), dict(tau=1e-45)):
        assert distill(**bad) == WIND_ERR_ARG, bad

    def lattice(e=p, e_t=64, pp=p, labels=p, frames=p, counts=p, B=2, T=4, U=2, loss=p, ws=p, size=1 << 40):
        return lib.wind_transducer_loss(C.byref(lay), e, 256, e_t, pp, 192, 64, labels, frames, counts, None, B, T, U, loss, None, None, None, None, ws, size, None)

    for bad in (dict(e=None), dict(e=p + 1), dict(e_t=-64), dict(pp=None), dict(labels=None), dict(frames=None), dict(counts=None), dict(B=0), dict(T=-1),
                dict(U=-1), dict(loss=None), dict(ws=None), dict(ws=p + 8), dict(size=16)):
        assert lattice(**bad) == WIND_ERR_ARG, bad


def test_python_functions_refuse_tensors_that_do_not_fit():
    from paper_2505_13765_amd import distill_loss, label_loss, transducer_loss

    h, w, lab = torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: label_loss(h, w, None, lab),                                        # not on a GPU
                 lambda: label_loss(h, w.half(), None, lab),
                 lambda: label_loss(h, w[0], None, lab),
                 lambda: label_loss(h, w, None, lab, grad=("x",)),
                 lambda: label_loss(h, w, None, lab, grad=("h", "h")),
                 lambda: label_loss(h[0], w, None, lab),
                 lambda: distill_loss(h, w, None, lab[:, None], None),
                 lambda: distill_loss(h, w, None, lab, torch.zeros(3, 1)),
                 lambda: transducer_loss(h, h, w, None, lab, lab, lab),
                 lambda: transducer_loss(h[None], h[None, :0], w, None, lab[None], lab, lab)):
        with pytest.raises(ValueError):
            call()
