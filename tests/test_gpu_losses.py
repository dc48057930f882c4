"""The losses over the output layer and their gradients against plain references in 64 bits (loss_reference.py, with the bounds' derivation)."""
import math

import pytest
import torch

from loss_reference import close, row_loss, transducer_loss

pytestmark = pytest.mark.gpu

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def api():
    import paper_2505_13765_amd as wind

    return wind


def rows(N, H, V1, dtype, seed, left_out=0.2, bias=True):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn((N, H), generator=g)
    w = torch.randn((V1, H), generator=g) / math.sqrt(H)
    b = 0.3 * torch.randn(V1, generator=g) if bias else None
    labels = torch.randint(0, V1, (N,), generator=g, dtype=torch.int32)
    labels[torch.rand(N, generator=g) < left_out] = -100
    h[labels < 0] = float("nan")          # what padding may hold
    weights = torch.rand(N, generator=g) - 0.2
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    return h.to(DTYPES[dtype]).cuda(), w.to(DTYPES[dtype]).cuda(), cuda(b), labels.cuda(), weights.cuda()


def check(got, ref, names):
    for name, t in zip(("loss",) + tuple(names), got):
        close(t, *ref[name], name)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("N,H,V1", [(0, 8, 5), (1, 1, 2), (1, 640, 1025), (5, 7, 33), (63, 64, 31), (64, 65, 32), (129, 100, 1025), (257, 640, 1000), (700, 33, 130)])
def test_label_loss(N, H, V1, dtype):
    wind = api()
    h, w, b, labels, weights = rows(N, H, V1, dtype, N + H)
    ref = row_loss(h, w, b, labels, weights=weights)
    check(wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b")), ref, "hwb")
    close(wind.label_loss(h, w, b, labels), *ref["loss"], "loss alone")
    (loss, db) = wind.label_loss(h, w, b, labels, weights, grad=("b",))
    close(db, *ref["b"], "b alone")


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("N,H,V1,K,tau", [(1, 8, 5, 1, 1.0), (40, 64, 33, 33, 0.5), (200, 100, 1025, 16, 2.0), (333, 65, 77, 5, 4.0), (70, 32, 2100, 1024, 1.0)])
def test_distill_loss(N, H, V1, K, tau, dtype):
    wind = api()
    h, w, b, _, weights = rows(N, H, V1, dtype, N + K, left_out=0.0)
    g = torch.Generator().manual_seed(N)
    labels = torch.randint(-1, V1, (N, K), generator=g, dtype=torch.int32)     # outputs named twice among them
    logits = 3 * torch.randn((N, K), generator=g)
    logits[torch.rand((N, K), generator=g) < 0.1] = -math.inf
    labels[N // 2] = -1                                                        # a row without entries
    logits[N // 3] = -math.inf                                                 # and one that a mask empties
    logits[N // 4] = torch.finfo(torch.float32).min                            # a mask of the type's lowest value leaves them equal
    labels, logits = labels.cuda(), logits.cuda()
    ref = row_loss(h, w, b, labels, logits, tau, weights)
    check(wind.distill_loss(h, w, b, labels, logits, tau, weights, grad=("h", "w", "b")), ref, "hwb")
    close(wind.distill_loss(h, w, b, labels, logits, tau), *ref["loss"], "loss alone")


@pytest.mark.parametrize("N,H,V1,K,dtype", [(2500, 40, 9000, 24, "bf16"), (1500, 33, 8193, 40, "f32"), (900, 96, 8200, 128, "bf16"), (20000, 24, 70, 3, "bf16")])
def test_many_teacher_logits(N, H, V1, K, dtype):
    """Entries enough to be sorted by column, with outputs that a row names twice or in all of its entries."""
    wind = api()
    h, w, b, _, weights = rows(N, H, V1, dtype, N, left_out=0.0)
    g = torch.Generator().manual_seed(N + 1)
    labels = torch.randint(-1, V1, (N, K), generator=g, dtype=torch.int32)
    labels[:, 1] = labels[:, 0]
    labels[::7, 2] = labels[::7, 0]
    labels[5] = V1 - 1
    labels[6] = -1
    logits = 2 * torch.randn((N, K), generator=g)
    labels, logits = labels.cuda(), logits.cuda()
    ref = row_loss(h, w, b, labels, logits, 2.0, weights)
    got = wind.distill_loss(h, w, b, labels, logits, 2.0, weights, grad=("h", "w", "b"))
    check(got, ref, "hwb")
    again = wind.distill_loss(h, w, b, labels, logits, 2.0, weights, grad=("h", "w", "b"))
    assert all(torch.equal(x, y) for x, y in zip(got, again))


def test_many_short_rows():
    """More rows than one launch counts, an odd number, most of them padding."""
    wind = api()
    h, w, b, labels, weights = rows(40961, 40, 50, "bf16", 15, left_out=0.7)
    ref = row_loss(h, w, b, labels, weights=weights)
    check(wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b")), ref, "hwb")


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_larger_tiles(dtype):
    """Shapes whose products take 128- and 256-wide tiles, ragged at every edge."""
    wind = api()
    for N, H, V1 in ((1500, 700, 1601), (4200, 1300, 4100)):
        h, w, b, labels, weights = rows(N, H, V1, dtype, N)
        ref = row_loss(h, w, b, labels, weights=weights)
        check(wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b")), ref, "hwb")
        del ref


def test_more_rows_than_a_chunk_holds():
    wind = api()
    N, H, V1 = 5000, 64, 65537
    h, w, b, labels, weights = rows(N, H, V1, "bf16", 9)
    ref = row_loss(h, w, b, labels, weights=weights)
    check(wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b")), ref, "hwb")
    labels[:4900] = -1                       # the later chunks hold nothing
    ref = row_loss(h, w, b, labels, weights=weights)
    check(wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b")), ref, "hwb")


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_no_row_counts(dtype):
    wind = api()
    h, w, b, labels, weights = rows(40, 48, 70, dtype, 1, left_out=2.0)
    loss, dh, dw, db = wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b"))
    for t in (loss, dh, dw, db):
        assert not t.any()


def test_labels_that_do_not_exist():
    wind = api()
    h, w, b, labels, weights = rows(50, 64, 40, "bf16", 2, left_out=0.0)
    labels[7], labels[8] = 40, 2 ** 31 - 1
    ref = row_loss(h, w, b, labels, weights=weights)
    got = wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b"))
    check(got, ref, "hwb")
    assert torch.isnan(got[0][7:9]).all() and not got[1][7:9].any()


def test_barred_outputs_and_infinite_losses():
    """-inf in the bias bars an output: probability zero, a row that wants it has an infinite loss and the others a finite one."""
    wind = api()
    h, w, b, labels, weights = rows(70, 64, 200, "f32", 3, left_out=0.0)
    b[64:128] = -math.inf                    # a whole block of columns
    labels[labels.ge(64) & labels.lt(128)] = 3
    labels[5] = 70
    ref = row_loss(h, w, b, labels, weights=weights)
    got = wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b"))
    check(got, ref, "hwb")
    assert got[0][5] == math.inf and torch.isfinite(got[0]).sum() == 69


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_strides_and_alignment(dtype):
    wind = api()
    for H, pad, first in ((64, 8, 0), (64, 3, 1), (40, 5, 3)):
        h, w, b, labels, weights = rows(90, H, 70, dtype, H + pad)
        ref = row_loss(h, w, b, labels, weights=weights)
        wide_h, wide_w = (torch.full((t.shape[0] * (H + pad) + first,), float("nan"), dtype=t.dtype, device="cuda") for t in (h, w))
        vh, vw = (t[first:].view(-1, H + pad)[:, :H] for t in (wide_h, wide_w))
        vh.copy_(h)
        vw.copy_(w)
        check(wind.label_loss(vh, vw, b, labels, weights, grad=("h", "w", "b")), ref, "hwb")
    check(wind.label_loss(h, w, None, labels, weights, grad=("h", "w", "b")), row_loss(h, w, None, labels, weights=weights), "hwb")


def lattice(B, T, U, H, V1, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    e, p = torch.randn((B, T, H), generator=g), torch.randn((B, U + 1, H), generator=g)
    w = torch.randn((V1, H), generator=g) / math.sqrt(H)
    b = 0.3 * torch.randn(V1, generator=g)
    b[-1] += 1.0
    labels = torch.randint(0, V1 - 1, (B, U), generator=g, dtype=torch.int32)
    frames = torch.randint(max(T // 2, min(T, 1)), T + 1, (B,), generator=g, dtype=torch.int32)
    counts = torch.randint(0, U + 1, (B,), generator=g, dtype=torch.int32)
    frames[0], counts[0] = T, U
    for i in range(B):                        # padding may hold anything
        e[i, int(frames[i]):] = float("nan")
        p[i, int(counts[i]) + 1:] = float("inf")
        labels[i, int(counts[i]):] = -7
    weights = torch.rand(B, generator=g) + 0.1
    dt = DTYPES[dtype]
    return [t.cuda() for t in (e.to(dt), p.to(dt), w.to(dt), b, labels, frames, counts, weights)]


GRAD = ("e", "p", "w", "b")


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("B,T,U,H,V1", [(1, 1, 0, 8, 2), (1, 1, 3, 8, 5), (2, 6, 0, 33, 9), (3, 9, 4, 64, 33), (5, 17, 11, 40, 70), (2, 3, 70, 32, 40), (70, 4, 3, 16, 12),
                                        (2, 40, 130, 24, 31), (3, 150, 5, 72, 1025), (40, 6, 30, 20, 17)])
def test_transducer_loss(B, T, U, H, V1, dtype):
    wind = api()
    a = lattice(B, T, U, H, V1, dtype, B + T + U)
    ref = transducer_loss(*a)
    check(wind.transducer_loss(*a, grad=GRAD), ref, GRAD)
    close(wind.transducer_loss(*a), *ref["loss"], "loss alone")
    check(wind.transducer_loss(*a, grad=("p",)), ref, ("p",))


@pytest.mark.parametrize("T,U", [(3, 1100), (2, 2200), (2, 4095)])
def test_long_transcripts(T, U):
    """More labels than a workgroup has threads: several cells per thread."""
    wind = api()
    a = lattice(2, T, U, 16, 12, "f32", U)
    check(wind.transducer_loss(*a, grad=GRAD), transducer_loss(*a), GRAD)


def test_improbable_transcripts():
    """Probabilities far below what fp32 holds, on single arcs and over the path."""
    wind = api()
    e, p, w, b, labels, frames, counts, weights = lattice(3, 30, 12, 32, 20, "f32", 4)
    b[:-1] -= 90.0                            # every label about e^-90
    ref = transducer_loss(e, p, w, b, labels, frames, counts, weights)
    assert float(ref["loss"][0][0]) > 1000
    check(wind.transducer_loss(e, p, w, b, labels, frames, counts, weights, grad=GRAD), ref, GRAD)


def test_utterances_that_do_not_count():
    """Without frames, with a label that does not exist, with blank as a label, of probability zero; lengths out of range are clamped."""
    wind = api()
    e, p, w, b, labels, frames, counts, weights = lattice(7, 8, 5, 32, 20, "bf16", 5)
    e, p = torch.nan_to_num(e), torch.nan_to_num(p, posinf=0.0)
    labels.clamp_(min=0)
    frames[:], counts[:] = 8, 5
    frames[1], labels[2, 3], labels[3, 0] = 0, -1, 19
    b[4] = -math.inf
    labels[labels == 4] = 5
    labels[4, 1] = 4
    frames[5], counts[6] = 99, 99
    frames[0] = -3
    ref = transducer_loss(e, p, w, b, labels, frames, counts, weights)
    got = wind.transducer_loss(e, p, w, b, labels, frames, counts, weights, grad=GRAD)
    check(got, ref, GRAD)
    assert got[0][:2].tolist() == [0.0, 0.0] and torch.isnan(got[0][2:4]).all() and got[0][4] == math.inf
    assert not got[1][:5].any() and not got[2][:5].any() and got[1][5:].any()


def test_no_utterance_counts():
    wind = api()
    a = lattice(3, 8, 5, 32, 20, "bf16", 6)
    a[5].zero_()
    for t in wind.transducer_loss(*a, grad=GRAD):
        assert not t.any()
    a = lattice(2, 0, 3, 32, 20, "f32", 6)    # no frame at all
    for t in wind.transducer_loss(*a, grad=GRAD):
        assert not t.any()


def test_lattice_strides():
    wind = api()
    e, p, *rest = lattice(4, 10, 6, 40, 30, "bf16", 7)
    ref = transducer_loss(e, p, *rest)
    flipped = e.transpose(0, 1).contiguous().transpose(0, 1)                    # time first
    wide = torch.full((4, 7, 43), float("nan"), dtype=p.dtype, device="cuda")
    wide[:, :, 1:41] = p
    check(wind.transducer_loss(flipped, wide[:, :, 1:41], *rest, grad=GRAD), ref, GRAD)
    one = p[:1].expand(4, 7, 40)                                                 # the same prediction rows for every utterance
    check(wind.transducer_loss(e, one, *rest, grad=GRAD), transducer_loss(e, torch.nan_to_num(one, posinf=0.0), *rest), GRAD)


def test_lattice_in_chunks():
    """More nodes than a chunk holds: frames and labels whose sums go over a chunk's end."""
    wind = api()
    e, p, w, b, labels, frames, counts, weights = lattice(16, 400, 60, 64, 1025, "bf16", 8)
    frames[:], counts[:] = 400, 60
    e, p, labels = torch.nan_to_num(e), torch.nan_to_num(p, posinf=0.0), labels.clamp(min=0)
    frames[3], counts[4] = 211, 17
    a = (e, p, w, b, labels, frames, counts, weights)
    check(wind.transducer_loss(*a, grad=GRAD), transducer_loss(*a), GRAD)


def test_a_large_lattice_in_one_chunk():
    wind = api()
    a = lattice(3, 203, 40, 701, 40, "bf16", 16)
    a[0], a[1] = torch.nan_to_num(a[0]), torch.nan_to_num(a[1], posinf=0.0)
    a[4] = a[4].clamp(min=0)
    a[5][1] = 0
    check(wind.transducer_loss(*a, grad=GRAD), transducer_loss(*a), GRAD)
    check(wind.transducer_loss(*a, grad=("e",)), transducer_loss(*a), ("e",))


def test_gradients_against_differences():
    """Along a random direction of every input, fp32.  A central difference over 2 s is off by the losses' own bounds over s, and by its truncation,
    which is that of the same difference of the reference."""
    wind = api()
    s = 2.0 ** -6
    a = lattice(4, 12, 6, 48, 40, "f32", 10)
    for i in (0, 1):
        a[i] = torch.nan_to_num(a[i], posinf=0.0)
    got, ref = wind.transducer_loss(*a, grad=GRAD), transducer_loss(*a)
    weights = a[7].double().cpu()
    g = torch.Generator().manual_seed(3)
    for k, i in zip(GRAD, range(4)):
        step = torch.randn(a[i].shape, generator=g)
        step = (step / step.norm()).cuda()
        mine, exact, bound = [], [], 0.0
        for sign in (1, -1):
            moved = list(a)
            moved[i] = a[i] + sign * s * step
            there = transducer_loss(*moved)["loss"]
            mine.append(float((wind.transducer_loss(*moved).double().cpu() * weights).sum()))
            exact.append(float((there[0] * weights).sum()))
            bound += float((there[1] * weights).sum()) / (2 * s)
        slope = lambda x: float((x.double() * step.double()).sum())  # noqa: E731
        truncation = abs((exact[0] - exact[1]) / (2 * s) - slope(ref[k][0]))
        bound += truncation + float((ref[k][1] * step.abs().double()).sum())
        assert bound < 0.05 * a[i].shape[0] and abs((mine[0] - mine[1]) / (2 * s) - slope(got[1 + GRAD.index(k)])) <= bound, (k, mine, bound)


def test_same_bits_every_time_on_other_streams_and_in_graphs():
    wind = api()
    h, w, b, labels, weights = rows(900, 160, 700, "bf16", 11)
    lat = lattice(6, 30, 9, 64, 50, "bf16", 12)
    calls = (lambda: wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b")), lambda: wind.transducer_loss(*lat, grad=GRAD))
    for call in calls:
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        side = [torch.cuda.Stream(), torch.cuda.Stream()]
        outs = []
        for st in side:                       # two calls at once, each with its own workspace
            with torch.cuda.stream(st):
                outs.append(call())
        torch.cuda.synchronize()
        for out in outs:
            assert all(torch.equal(x, y) for x, y in zip(want, out))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = call()
        for _ in range(3):
            for t in held:
                t.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(want, held))
            again = call()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(want, again))


def test_a_graph_takes_what_its_inputs_hold_at_replay():
    """Other labels, other lengths, other numbers of rows that count."""
    wind = api()
    h, w, b, labels, weights = rows(700, 96, 300, "bf16", 13, left_out=0.0)
    graph = torch.cuda.CUDAGraph()
    wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b"))
    with torch.cuda.graph(graph):
        held = wind.label_loss(h, w, b, labels, weights, grad=("h", "w", "b"))
    for part in (0, 650, 700, 300):
        labels.copy_(torch.randint(0, 300, (700,), device="cuda", dtype=torch.int32))
        labels[:part] = -1
        graph.replay()
        torch.cuda.synchronize()
        check(held, row_loss(h, w, b, labels, weights=weights), "hwb")


def test_workspace_and_outputs_of_any_content():
    """The C entry point on buffers full of NaN: nothing is read before it is written, and nothing behind the outputs is touched."""
    import ctypes as C

    from paper_2505_13765_amd.binding import OutputLayer, load_library

    lib = load_library()
    h, w, b, labels, weights = rows(300, 72, 90, "bf16", 14)
    lay = OutputLayer(w.data_ptr(), b.data_ptr(), 72, 90, 72, 1)
    n = C.c_size_t(0)
    assert lib.wind_row_loss_workspace_bytes(C.byref(lay), 300, 1, 1, C.byref(n)) == 0
    ref = row_loss(h, w, b, labels, weights=weights)
    ws = torch.full((n.value,), 0xFF, dtype=torch.uint8, device="cuda")
    outs = [torch.full((size + 64,), float("nan"), dtype=dt, device="cuda")
            for size, dt in ((300, torch.float32), (300 * 72, torch.bfloat16), (90 * 72, torch.bfloat16), (90, torch.float32))]
    assert lib.wind_label_loss(C.byref(lay), h.data_ptr(), 72, labels.data_ptr(), weights.data_ptr(), 300, *(t.data_ptr() for t in outs), ws.data_ptr(), n.value,
                               torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    for t, shape, name in zip(outs, ((300,), (300, 72), (90, 72), (90,)), ("loss", "h", "w", "b")):
        assert torch.isnan(t[-64:].float()).all()
        close(t[:-64].view(shape), *ref[name], name)


def test_a_training_step_of_a_joiner():
    """As the three are used together: transducer loss of a batch, distillation of single frames from a teacher's scores as the beam search's
    scoring step returns them, and the prediction network's label loss, all on one output layer, whose gradients add up."""
    import numpy as np

    import wind_inputs as wi

    wind = api()
    cfg = wi.CONFIGS["tiny"]
    weights = wi.make_weights(cfg)
    teacher = wind.WindModel.from_config(cfg, weights)
    H, V1, K = cfg.Hj, cfg.V + 1, 6
    g = torch.Generator().manual_seed(1)
    f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()  # noqa: E731
    w_enc, b_enc, w_pred, b_pred, w_out, b_out = (f32(weights[k]) for k in ("w_enc", "b_enc", "w_pred", "b_pred", "w_out", "b_out"))
    frames = torch.randn((2, 20, cfg.D), generator=g).cuda()
    hidden = (0.5 * torch.randn((2, 6, cfg.Hp), generator=g)).cuda()
    e, p = frames @ w_enc.t() + b_enc, hidden @ w_pred.t() + b_pred
    student = w_out + 0.05 * torch.randn(w_out.shape, generator=g).cuda()
    labels = torch.randint(0, cfg.V, (2, 5), generator=g, dtype=torch.int32).cuda()
    lengths, counts = torch.tensor([20, 14], dtype=torch.int32).cuda(), torch.tensor([5, 3], dtype=torch.int32).cuda()
    # the teacher's scores of one frame for six hypotheses: log probabilities of its K best outputs (-1 where it has fewer)
    at, jumps, scores = (torch.zeros((6, K), dtype=dt, device="cuda") for dt in (torch.int32, torch.int32, torch.float32))
    teacher.beam_window_scores(frames[0, :1].contiguous(), hidden[0].contiguous(), K, out=(at, jumps, scores))
    z = torch.relu(e[0, :1] + p[0])
    a = wind.transducer_loss(e, p, student, b_out, labels, lengths, counts, grad=GRAD)
    d = wind.distill_loss(z, student, b_out, at, scores, grad=("h", "w", "b"))
    next_label = torch.cat([labels[0], labels.new_full((1,), -1)])
    c = wind.label_loss(z, student, b_out, next_label, grad=("h", "w", "b"))
    check(a, transducer_loss(e, p, student, b_out, labels, lengths, counts), GRAD)
    check(d, row_loss(z, student, b_out, at, scores), "hwb")
    check(c, row_loss(z, student, b_out, next_label), "hwb")
    # the teacher itself is at distance (almost) zero from what its largest logits keep: K of its outputs hold that share of its probability
    own = wind.distill_loss(z, w_out, b_out, at, scores)
    kept = torch.where(at >= 0, scores.double().exp(), 0.0).sum(1)
    assert torch.allclose(own.double(), -kept.log(), atol=1e-4)
    dw, db = a[3] + d[2] + c[2], a[4] + d[3] + c[3]
    assert torch.isfinite(dw).all() and torch.isfinite(db).all()
    with torch.no_grad():                    # and the step: the updated layer goes into a model that decodes
        student -= 0.01 * dw
        bias = b_out - 0.01 * db
    trained = dict(weights, w_out=student.cpu().numpy(), b_out=bias.cpu().numpy())
    model = wind.WindModel.from_config(cfg, trained)
    tokens, _ = model.decode(frames, lengths, 4, cfg.S)
    assert len(tokens) == 2
    model.close()
    teacher.close()


@pytest.mark.parametrize("N", (1, 13, 128))
def test_gradients_of_few_rows_are_only_rounded_once(N):
    """bf16 gradients of few rows: off by the result's own rounding (half a step, 2^-8 relative) and what dx on 16 bits leaves, not by a rounding of dx to 8 bits.

    dx_v = c (p_v - [v = label]) is kept to 2^-16 of itself, p_v to its logit's error, at most (H + 2) 2^-24 sum |h w| with the bias (one rounding a term) and twice that for
    the norm's, and 2^-20 for the functions and sums; products add (terms + 8) 2^-24 of their terms' sum.  The weight 1 + 2^-8 lies between two bf16 values: rounded to 8 bits, the
    label's dx alone, which is almost all of the gradient, would be off by 2^-8."""
    wind, H, V1 = api(), 64, 400
    g = torch.Generator().manual_seed(N)
    h, w = (0.25 * torch.randn(s, H, generator=g) for s in (N, V1))
    b, labels = 0.1 * torch.randn(V1, generator=g), torch.randint(0, V1, (N,), generator=g, dtype=torch.int32)
    h, w, c = h.bfloat16(), w.bfloat16(), 1 + 2.0**-8
    _, dh, dw = wind.label_loss(h.cuda(), w.cuda(), b.cuda(), labels.cuda(), weights=torch.full((N,), c).cuda(), grad=("h", "w"))
    h, w, b = h.double(), w.double(), b.double()
    p = torch.softmax(h @ w.T + b, dim=1)
    dx = c * (p - torch.nn.functional.one_hot(labels.long(), V1))
    logit = 2 * (H + 2) * 2.0**-24 * (h.abs() @ w.abs().T + b.abs()).amax(1, keepdim=True) + 2.0**-20
    off = 2.0**-16 * dx.abs() + c * p * logit
    for got, ref, bound in ((dh, dx @ w, off @ w.abs() + (V1 + 8) * 2.0**-24 * (dx.abs() @ w.abs())), (dw, dx.T @ h, off.T @ h.abs() + (N + 8) * 2.0**-24 * (dx.abs().T @ h.abs()))):
        err = (got.double().cpu() - ref).abs()
        assert (err <= 2.0**-8 * (ref.abs() + bound) + bound + 2.0**-133).all(), (err - 2.0**-8 * ref.abs()).max()
