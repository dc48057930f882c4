"""What the losses over the output layer take and refuse, and the workspaces they ask for, without a GPU."""
import ctypes as C

import pytest

from test_losses_cpu import lattice_size, layer, lib, rows_size  # noqa: F401  (lib: the fixture)


@pytest.mark.parametrize("V1,H,dtype,N", [(65537, 640, 1, 100000), (65537, 2048, 1, 40000), (50257, 768, 1, 131072), (128256, 4096, 1, 65536), (4097, 640, 1, 900000),
                                          (4097, 640, 1, 1000000), (65537, 2048, 0, 40000), (33, 48, 1, 50000000), (2, 1, 1, (1 << 31) - 1)])
def test_scores_of_many_rows_are_taken(lib, V1, H, dtype, N):  # noqa: F811
    """Whatever a step takes, with less memory than the step."""
    from paper_2505_13765_amd.binding import WIND_OK

    lay = layer(V1=V1, H=H, dtype=dtype)
    step, scores = rows_size(lib, lay, N), rows_size(lib, lay, N, grads=0)
    assert step[0] == scores[0] == WIND_OK and scores[1] <= step[1]


@pytest.mark.parametrize("V1,H,dtype,B,T,U", [(8193, 640, 1, 16, 750, 120), (4097, 200, 1, 32, 750, 120), (8193, 48, 1, 32, 750, 120), (8193, 640, 1, 32, 250, 40),
                                              (1025, 64, 1, 32, 750, 120), (8193, 640, 0, 32, 750, 120), (4097, 640, 1, 16, 750, 120)])
def test_scores_of_many_nodes_are_taken(lib, V1, H, dtype, B, T, U):  # noqa: F811
    from paper_2505_13765_amd.binding import WIND_OK

    lay = layer(V1=V1, H=H, dtype=dtype)
    step, scores = lattice_size(lib, lay, B, T, U), lattice_size(lib, lay, B, T, U, grads=0)
    assert step[0] == scores[0] == WIND_OK and scores[1] <= step[1]


@pytest.mark.parametrize("grads", (0, 1))
@pytest.mark.parametrize("V1,H,K", [(65537, 64, 1), (1 << 20, 64, 1), (1025, 640, 1024), (33, 32, 1024)])
def test_workspaces_hold_a_piece(lib, V1, H, K, grads):  # noqa: F811
    """Rows, statistics and entries of a piece, not of all rows: some bytes a row are all that a workspace grows by."""
    few, many = (rows_size(lib, layer(V1=V1, H=H, dtype=1), N, K=K, grads=grads)[1] for N in (1 << 22, 1 << 23))
    assert many < 4 << 30 and many - few <= 8 << 22


def test_widths_out_of_range_are_refused(lib):  # noqa: F811
    from paper_2505_13765_amd.binding import WIND_ERR_UNSUPPORTED, WIND_OK

    most = (1 << 23) - 32
    for grads in (0, 1):
        assert rows_size(lib, layer(V1=most, H=32), 8, grads=grads)[0] == WIND_OK
        assert rows_size(lib, layer(V1=32, H=most), 8, grads=grads)[0] == WIND_OK
        for bad in (dict(V1=most + 1, H=32), dict(V1=32, H=most + 1)):
            assert rows_size(lib, layer(**bad), 8, grads=grads)[0] == WIND_ERR_UNSUPPORTED and b"2^23" in lib.wind_last_error()
            assert lattice_size(lib, layer(**bad), 1, 4, 2, grads=grads)[0] == WIND_ERR_UNSUPPORTED


@pytest.mark.parametrize("V1,H,dtype,K", [(65537, 48, 1, 1), (65537, 2048, 1, 1), (4097, 640, 1, 16), (1025, 640, 0, 64), (33, 64, 0, 1), (8193, 1024, 1, 16), (50, 40, 1, 3)])
def test_a_workspace_for_many_rows_serves_fewer(lib, V1, H, dtype, K):  # noqa: F811
    """Also across the sizes where tiles, parts of sums, chunks and the sorting of entries change; and one for steps serves scores."""
    lay, last = layer(V1=V1, H=H, dtype=dtype), 0
    sizes = sorted({max(0, int(2 ** (x / 16)) + d) for x in range(0, 350) for d in (-1, 0, 1)} | set(range(9000, 12000, 64)))
    for N in sizes:
        need = rows_size(lib, lay, N, K=K)[1]
        assert need >= last, N
        assert rows_size(lib, lay, N, K=K, grads=0)[1] <= need
        last = need


@pytest.mark.parametrize("V1,H,dtype", [(1025, 640, 1), (33, 64, 0), (4097, 640, 1), (5000, 200, 0)])
def test_a_workspace_for_large_lattices_serves_smaller(lib, V1, H, dtype):  # noqa: F811
    lay = layer(V1=V1, H=H, dtype=dtype)
    steps = [0, 1, 2, 3, 7, 16, 17, 40, 63, 64, 65, 127, 128, 250, 256, 257, 700, 1023, 1024, 1100]
    for grads in (0, 1):
        for size in (lambda x: (x + 1, 250, 40), lambda x: (16, x, 40), lambda x: (3, 300, x), lambda x: (2, x, 1100), lambda x: (16, 2 * x, x // 4)):
            needs = [lattice_size(lib, lay, *size(x), grads=grads)[1] for x in steps]
            assert needs == sorted(needs), needs
    assert all(lattice_size(lib, lay, b, 250, 40, grads=0)[1] <= lattice_size(lib, lay, b, 250, 40)[1] for b in range(1, 40))


def test_widths_near_the_integers_end_are_refused(lib):  # noqa: F811
    """Rounding them up to whole panels must not leave the integers' range."""
    from paper_2505_13765_amd.binding import WIND_ERR_UNSUPPORTED

    for top in ((1 << 31) - 1, (1 << 31) - 31, (1 << 31) - 32):
        for bad in (dict(V1=top, H=1, stride=1), dict(V1=2, H=top)):
            assert rows_size(lib, layer(**bad), 8)[0] == WIND_ERR_UNSUPPORTED, bad
            assert lattice_size(lib, layer(**bad), 1, 4, 2)[0] == WIND_ERR_UNSUPPORTED, bad


@pytest.mark.parametrize("tau", (4e-39, 4.2e-39, 3e-39))
def test_temperatures_whose_scale_overflows_are_refused(lib, tau):  # noqa: F811
    """log2(e) / tau is what logits are multiplied with.  The buffers are made up: the call must not get further than its arguments."""
    from paper_2505_13765_amd.binding import WIND_ERR_ARG

    assert lib.wind_distill_loss(C.byref(layer()), 4096, 64, 4096, 4096, 2, tau, None, 8, 4096, None, None, None, 4096 + 1, 1 << 40, None) == WIND_ERR_ARG
    assert b"temperature" in lib.wind_last_error()


def test_lattices_whose_launches_would_not_fit_are_refused(lib):  # noqa: F811
    """A launch has fewer than 2^32 threads: the sums of a gradient's frames and prediction rows take 256 for each 256 columns of one.  Scores have none."""
    from paper_2505_13765_amd.binding import WIND_ERR_UNSUPPORTED, WIND_OK

    for lay, most in ((layer(V1=33, H=640), ((1 << 24) - 2048 - 3) // 3), (layer(V1=33, H=64), (1 << 24) - 2048 - 4)):
        for B in (1, 8):
            T = most // B - 2
            assert lattice_size(lib, lay, B, T, 1)[0] == WIND_OK
            assert lattice_size(lib, lay, B, T + 2, 1)[0] == WIND_ERR_UNSUPPORTED and b"2^24" in lib.wind_last_error()
            assert lattice_size(lib, lay, B, T + 2, 1, grads=0)[0] == WIND_OK
    assert lattice_size(lib, layer(), 1 << 25, 1, 0, grads=0)[0] == WIND_ERR_UNSUPPORTED     # 64 threads for each recursion
    assert lattice_size(lib, layer(), (1 << 25) - 1, 1, 0, grads=0)[0] == WIND_OK


def test_losses_without_a_graph_are_not_taken_for_ones_with():
    """Where autograd would expect a graph (no gradients asked for, an input that requires them), the call says that there is none; with gradients asked for, or outside
    autograd's recording, it goes on (here: to the next refusal, no GPU)."""
    import torch

    from paper_2505_13765_amd import distill_loss, label_loss, transducer_loss

    h, w, lab = torch.zeros(3, 4), torch.zeros(5, 4), torch.zeros(3, dtype=torch.int32)
    leaf = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = (lambda f, **k: label_loss(f(h), w, None, lab, **k), lambda f, **k: label_loss(h, f(w), None, lab, **k),
             lambda f, **k: label_loss(h, w, f(torch.zeros(5)), lab, **k), lambda f, **k: label_loss(h, w, None, lab, weights=f(torch.ones(3)), **k),
             lambda f, **k: distill_loss(h, w, None, lab[:, None], f(torch.zeros(3, 1)), **k),
             lambda f, **k: transducer_loss(f(h[None]), h[None], w, None, lab[None, :2], lab[:1], lab[:1], **k),
             lambda f, **k: transducer_loss(h[None], f(h[None]), w, None, lab[None, :2], lab[:1], lab[:1], **k))
    for call in calls:
        with pytest.raises(ValueError, match="no autograd graph"):
            call(leaf)
        for go_on in (lambda: call(leaf, grad=("w",)), lambda: call(lambda t: t)):
            with pytest.raises(ValueError, match="GPU"):
                go_on()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call(leaf)
