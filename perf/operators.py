"""What is timed when the speed of the training losses over the output layer is followed: single calls of `label_loss`,
`distill_loss` and `transducer_loss` on tensors that a training or scoring program has on the GPU.

`run` computes them in plain torch operations (32 bits, the lattice's sums in 64), or, with `own` set, through the library.
`exact` is the same from the definitions in 64 bits.  V1 counts the outputs: the labels and, in the last column, blank.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# kind "label": cross entropy of N rows | "distill": of N rows against K logits of a teacher | "transducer": of B utterances of up to T frames
# and U labels.  left_out: share of the rows that carry no label (padding).  grad: a training step, else scores alone.


def listed():
    return [
        # scores of a window's rows for a few hypotheses: the smallest call that a search makes
        {"name": "label_scores", "kind": "label", "N": 16, "H": 640, "V1": 1025, "dtype": "bf16", "left_out": 0.0, "grad": False},
        # the prediction network trained as a language model on a padded batch of transcripts
        {"name": "label_step", "kind": "label", "N": 8192, "H": 640, "V1": 4097, "dtype": "bf16", "left_out": 0.3, "grad": True},
        # the same over a vocabulary of words
        {"name": "label_words", "kind": "label", "N": 8192, "H": 2048, "V1": 65537, "dtype": "bf16", "left_out": 0.1, "grad": True},
        # fp32 weights, odd sizes
        {"name": "label_f32", "kind": "label", "N": 1237, "H": 320, "V1": 1025, "dtype": "f32", "left_out": 0.1, "grad": True},
        # a student's distance from its teacher on one short utterance
        {"name": "distill_scores", "kind": "distill", "N": 61, "K": 8, "H": 640, "V1": 1025, "dtype": "bf16", "left_out": 0.0, "grad": False},
        # a step on the joiner rows of a batch, few teacher logits of a large vocabulary
        {"name": "distill_step", "kind": "distill", "N": 12000, "K": 16, "H": 1024, "V1": 8193, "dtype": "bf16", "left_out": 0.2, "grad": True},
        # many teacher logits, fp32 weights
        {"name": "distill_f32", "kind": "distill", "N": 3001, "K": 64, "H": 640, "V1": 1025, "dtype": "f32", "left_out": 0.0, "grad": True},
        # the probability of one transcript of ten seconds
        {"name": "transducer_score", "kind": "transducer", "B": 1, "T": 125, "U": 20, "H": 640, "V1": 1025, "dtype": "bf16", "grad": False},
        # the smallest model, fp32
        {"name": "transducer_tiny", "kind": "transducer", "B": 4, "T": 64, "U": 12, "H": 64, "V1": 33, "dtype": "f32", "grad": True},
        # training steps: a batch of short utterances, and one of long ones over a larger vocabulary
        {"name": "transducer_step", "kind": "transducer", "B": 32, "T": 250, "U": 40, "H": 640, "V1": 1025, "dtype": "bf16", "grad": True},
        {"name": "transducer_long", "kind": "transducer", "B": 16, "T": 750, "U": 120, "H": 640, "V1": 4097, "dtype": "bf16", "grad": True},
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], even over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    while True:
        kind = rng.choice(("label", "distill", "transducer"))
        case = {"kind": kind, "H": _log_int(rng, 48, 2048), "dtype": rng.choice(("bf16", "bf16", "f32")), "grad": rng.random() < 0.75}
        if kind == "transducer":
            case |= {"B": _log_int(rng, 1, 32), "T": _log_int(rng, 8, 750), "U": _log_int(rng, 1, 120), "V1": _log_int(rng, 33, 8193)}
        else:
            case |= {"N": _log_int(rng, 1, 16384), "V1": _log_int(rng, 33, 65537), "left_out": rng.choice((0.0, 0.1, 0.5))}
        if kind == "distill":
            case["K"] = min(case["V1"], _log_int(rng, 1, 64))
        if work(case)["flops"] <= (1e12 if case["dtype"] == "f32" else 6e12):
            return case


def _lengths(case, g):
    """Frames and labels of every utterance: from half of the largest up, the first of full length."""
    lo = [(n + 1) // 2 for n in (case["T"], case["U"])]
    T, U = (torch.randint(a, n + 1, (case["B"],), generator=g) for a, n in zip(lo, (case["T"], case["U"])))
    T[0], U[0] = case["T"], case["U"]
    return T, U


def _rows(case):
    """Rows that are computed, as work() counts them."""
    if case["kind"] != "transducer":
        return case["N"] * (1.0 - case["left_out"])
    B = case["B"]
    return case["T"] * (case["U"] + 1) + (B - 1) * 0.75 * case["T"] * (0.75 * case["U"] + 1)


def work(case):
    H, V1, n = case["H"], case["V1"], _rows(case)
    size = 2 if case["dtype"] == "bf16" else 4
    inputs = case["B"] * (0.75 * (case["T"] + case["U"]) + 1) * H if case["kind"] == "transducer" else n * H
    move = (V1 * H + inputs) * size + 4 * V1
    rows = 4 * n if case["kind"] != "transducer" else 0
    teacher = 8 * n * case["K"] if case["kind"] == "distill" else 4 * n if case["kind"] == "label" else 4 * case["B"] * case["U"]
    times = 3 if case["grad"] else 1   # logits; with gradients also their products with the weights and with the rows
    return {"bytes": move * (2 if case["grad"] else 1) + rows + teacher, "flops": times * 2.0 * n * H * V1}


def prepare(case, seed):
    g = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device="cuda").manual_seed(seed)
    H, V1 = case["H"], case["V1"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    normal = lambda *shape: torch.randn(shape, generator=gd, device="cuda")  # noqa: E731
    w = normal(V1, H) / math.sqrt(H)
    s = {"case": case, "w": w.to(dtype), "b": 0.1 * normal(V1)}
    if case["kind"] == "transducer":
        B, T, U = case["B"], case["T"], case["U"]
        frames, counts = _lengths(case, g)
        # blank wins most nodes, as after some training
        s["b"][-1] += math.log(V1) + 1.0
        labels = torch.randint(0, V1 - 1, (B, U), generator=gd, device="cuda", dtype=torch.int32)
        p = normal(B, U + 1, H)
        p[:, :U] += 3.0 * w[labels.long()]
        s |= {"e": normal(B, T, H).to(dtype), "p": p.to(dtype), "labels": labels, "frames": frames.int().cuda(), "counts": counts.int().cuda(),
              "weights": torch.full((B,), 1.0 / B, device="cuda")}
        return s
    N = case["N"]
    labels = torch.randint(0, V1, (N,), generator=gd, device="cuda", dtype=torch.int32)
    h = normal(N, H) + 4.0 * w[labels.long()]
    out = torch.rand((N,), generator=gd, device="cuda") < case["left_out"]
    s["h"] = h.to(dtype)
    if case["kind"] == "label":
        s["labels"] = torch.where(out, -1, labels)
        s["weights"] = torch.full((N,), 1.0 / max(N, 1), device="cuda")
        return s
    # the teacher's largest logits: distinct labels, the true one first
    K = case["K"]
    step = 1 + torch.randint(0, max(1, (V1 - 1) // K), (N, 1), generator=gd, device="cuda")
    at = (labels[:, None].long() + step * torch.arange(K, device="cuda")) % V1
    s["at"] = torch.where(out[:, None], -1, at).int().contiguous()
    s["logits"] = (4.0 * normal(N, K).abs().neg() + 4.0).sort(dim=1, descending=True)[0].contiguous()
    s["weights"] = (0.5 + torch.rand((N,), generator=gd, device="cuda")) / max(N, 1)
    s["temperature"] = 2.0
    return s


def run(state):
    case = state["case"]
    if own:
        import paper_2505_13765_amd as wind

        grad = None if not case["grad"] else ("e", "p", "w", "b") if case["kind"] == "transducer" else ("h", "w", "b")
        if case["kind"] == "label":
            return wind.label_loss(state["h"], state["w"], state["b"], state["labels"], weights=state["weights"], grad=grad)
        if case["kind"] == "distill":
            return wind.distill_loss(state["h"], state["w"], state["b"], state["at"], state["logits"], temperature=state["temperature"],
                                     weights=state["weights"], grad=grad)
        return wind.transducer_loss(state["e"], state["p"], state["w"], state["b"], state["labels"], state["frames"], state["counts"],
                                    weights=state["weights"], grad=grad)
    return {"label": _label, "distill": _distill, "transducer": _transducer}[case["kind"]](state)


def _log_norm(x):
    top = x.amax(dim=1, keepdim=True)
    return top + (x - top).exp().sum(dim=1, keepdim=True).log()


def _label(s):
    h, w, kept = s["h"].float(), s["w"].float(), s["labels"] >= 0
    at = s["labels"].long().clamp(min=0)[:, None]
    x = h @ w.T + s["b"]
    norm = _log_norm(x)
    loss = torch.where(kept, (norm - x.gather(1, at))[:, 0], 0.0)
    if not s["case"]["grad"]:
        return loss
    scale = torch.where(kept, s["weights"], 0.0)[:, None]
    d = (x - norm).exp() * scale
    d.scatter_add_(1, at, -scale)
    return loss, (d @ w).to(s["h"].dtype), (d.T @ h).to(s["w"].dtype), d.sum(dim=0)


def _distill(s):
    h, w, t = s["h"].float(), s["w"].float(), s["temperature"]
    there = s["at"] >= 0
    kept = there.any(dim=1)
    at = s["at"].long().clamp(min=0)
    teacher = torch.where(there, s["logits"] / t, -math.inf)
    teacher = torch.where(kept[:, None], teacher, 0.0)
    log_q = teacher - _log_norm(teacher)
    q = torch.where(there, log_q.exp(), 0.0)
    x = (h @ w.T + s["b"]) / t
    norm = _log_norm(x)
    terms = torch.where(q > 0, q * (log_q - x.gather(1, at) + norm), 0.0)
    loss = t * t * terms.sum(dim=1)
    if not s["case"]["grad"]:
        return loss
    scale = torch.where(kept, t * s["weights"], 0.0)[:, None]
    d = (x - norm).exp() * scale
    d.scatter_add_(1, at, -scale * q)
    return loss, (d @ w).to(s["h"].dtype), (d.T @ h).to(s["w"].dtype), d.sum(dim=0)


def _transducer(s):
    e, p, w, V1 = s["e"].float(), s["p"].float(), s["w"].float(), s["case"]["V1"]
    (B, T, _), U1 = e.shape, p.shape[1]
    frames, counts = s["frames"].long(), s["counts"].long()
    t, u = torch.arange(T, device="cuda"), torch.arange(U1, device="cuda")
    b_at, t_at, u_at = ((t < frames[:, None])[:, :, None] & (u <= counts[:, None])[:, None, :]).nonzero(as_tuple=True)
    z = torch.relu(e[b_at, t_at] + p[b_at, u_at])
    x = z @ w.T + s["b"]
    norm = _log_norm(x)
    padded = torch.cat((s["labels"].long(), s["labels"].new_zeros((B, 1)).long()), dim=1)
    label = padded[b_at, u_at][:, None]
    stop = u_at == counts[b_at]
    # log probabilities of the nodes in 64 bits: blank, and the next label (behind the last one: 0, which no path takes)
    blank, emit = (torch.zeros((B, T, U1), dtype=torch.float64, device="cuda") for _ in range(2))
    blank[b_at, t_at, u_at] = (x[:, -1:] - norm)[:, 0].double()
    emit[b_at, t_at, u_at] = torch.where(stop, 0.0, (x.gather(1, label) - norm)[:, 0].double())
    run_up = emit.cumsum(dim=2) - emit   # labels emitted on one frame before u
    alpha = [run_up[:, 0]]
    for i in range(1, T):
        alpha.append(run_up[:, i] + torch.logcumsumexp(alpha[-1] + blank[:, i - 1] - run_up[:, i], dim=1))
    alpha = torch.stack(alpha, dim=1)
    every, last = torch.arange(B, device="cuda"), frames - 1
    total = (alpha + blank)[every, last, counts]
    if not s["case"]["grad"]:
        return (-total).float()
    beyond = u > counts[:, None]
    after = torch.where(u == counts[:, None], 0.0, -math.inf).double()   # log probability of the end, behind the last frame
    beta = [after]
    for i in range(T - 1, -1, -1):
        here = (torch.where((i < frames)[:, None], beta[-1] + blank[:, i], -math.inf) + run_up[:, i]).masked_fill(beyond, -math.inf)
        here = torch.logcumsumexp(here.flip(1), dim=1).flip(1) - run_up[:, i]
        beta.append(torch.where((i < frames)[:, None], here, after))
    beta = torch.stack(beta[::-1], dim=1)
    weight = s["weights"][b_at].double()
    start = (alpha - total[:, None, None])[b_at, t_at, u_at]
    to_blank = weight * (start + blank[b_at, t_at, u_at] + beta[b_at, t_at + 1, u_at]).exp()
    to_label = weight * torch.where(stop, 0.0, (start + emit[b_at, t_at, u_at] + beta[b_at, t_at, (u_at + 1).clamp(max=U1 - 1)]).exp())
    d = (x - norm).exp() * (to_blank + to_label).float()[:, None]
    d[:, -1] -= to_blank.float()
    d.scatter_add_(1, label, -to_label.float()[:, None])
    dz = torch.where(z > 0, d @ w, 0.0)
    de = torch.zeros((B * T, dz.shape[1]), device="cuda").index_add_(0, b_at * T + t_at, dz).view_as(e)
    dp = torch.zeros((B * U1, dz.shape[1]), device="cuda").index_add_(0, b_at * U1 + u_at, dz).view_as(p)
    return (-total).float(), de.to(s["e"].dtype), dp.to(s["p"].dtype), (d.T @ z).to(s["w"].dtype), d.sum(dim=0)


def exact(case, seed):
    s = prepare(case, seed)
    w, b = s["w"].double(), s["b"].double()
    if case["kind"] == "transducer":
        return _exact_transducer(s, w, b)
    h = s["h"].double()
    tau = s.get("temperature", 1.0)
    log_p = torch.log_softmax(torch.addmm(b, h, w.t()) / tau, dim=1)
    # the targets as a distribution over all outputs (a row without any: zeros)
    q = torch.zeros_like(log_p)
    if case["kind"] == "label":
        rows = torch.nonzero(s["labels"] >= 0)[:, 0]
        q[rows, s["labels"][rows].long()] = 1.0
    else:
        rows = torch.nonzero(s["at"][:, 0] >= 0)[:, 0]
        share = torch.softmax(s["logits"][rows].double() / tau, dim=1)
        q[rows[:, None], s["at"][rows].long()] = share
    loss = tau * tau * (torch.xlogy(q, q) - q * log_p).sum(dim=1)
    if not case["grad"]:
        return loss
    d = log_p.exp_()
    d *= q.sum(dim=1, keepdim=True)
    d -= q
    d *= tau * s["weights"].double()[:, None]
    return loss, torch.mm(d, w), torch.mm(d.t(), h), d.sum(dim=0)


def _exact_transducer(s, w, b):
    """Utterance by utterance, the lattice cell by diagonal on the host, the gradient from the nodes' expected counts."""
    out, dw, db = {k: [] for k in ("loss", "e", "p")}, torch.zeros_like(w), torch.zeros_like(b)
    for i in range(s["case"]["B"]):
        T, U = int(s["frames"][i]), int(s["counts"][i])
        e, p, y = s["e"][i].double(), s["p"][i].double(), s["labels"][i, :U].long()
        z = (e[:T, None] + p[None, :U + 1]).clamp(min=0.0)
        log_p = torch.log_softmax(torch.matmul(z, w.t()) + b, dim=2)
        stay = log_p[:, :, -1].cpu().numpy()
        take = np.full((T, U + 1), -np.inf)
        take[:, :U] = log_p[:, torch.arange(U, device="cuda"), y].cpu().numpy()
        ahead, back = np.full((T + 1, U + 2), -np.inf), np.full((T + 1, U + 2), -np.inf)   # cell (t, u) of ahead sits at [t + 1, u + 1]
        ahead[1, 1], back[T, U] = 0.0, 0.0
        for d in range(1, T + U):
            t = np.arange(max(0, d - U), min(T - 1, d) + 1)
            u = d - t
            down = np.where(t > 0, ahead[t, u + 1] + stay[t - 1, u], -np.inf)
            right = np.where(u > 0, ahead[t + 1, u] + take[t, u - 1], -np.inf)
            ahead[t + 1, u + 1] = np.logaddexp(down, right)
        for d in range(T + U - 1, -1, -1):
            t = np.arange(max(0, d - U), min(T - 1, d) + 1)
            u = d - t
            back[t, u] = np.logaddexp(back[t + 1, u] + stay[t, u], back[t, u + 1] + take[t, u])
        out["loss"].append(-back[0, 0])
        if not s["case"]["grad"]:
            continue
        here = ahead[1:, 1:] - back[0, 0]
        weight = float(s["weights"][i])
        by_blank = torch.from_numpy(weight * np.exp(here + stay + back[1:, :U + 1])).cuda()
        by_label = torch.from_numpy(weight * np.exp(here + take + back[:T, 1:])).cuda()
        d = log_p.exp_() * (by_blank + by_label)[:, :, None]
        d[:, :, -1] -= by_blank
        d[:, torch.arange(U, device="cuda"), y] -= by_label[:, :U]
        dz = torch.matmul(d, w) * (z > 0)
        de, dp = torch.zeros_like(e), torch.zeros_like(p)
        de[:T], dp[:U + 1] = dz.sum(dim=1), dz.sum(dim=0)
        out["e"].append(de)
        out["p"].append(dp)
        dw += torch.mm(d.flatten(0, 1).t(), z.flatten(0, 1))
        db += d.sum(dim=(0, 1))
    loss = torch.tensor(out["loss"], dtype=torch.float64)
    return (loss, torch.stack(out["e"]), torch.stack(out["p"]), dw, db) if s["case"]["grad"] else loss
