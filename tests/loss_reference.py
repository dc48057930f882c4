"""Plain references in 64 bits for the losses over the output layer, and how far fp32 sums and bf16 roundings can be from them.

Bounds.  u = 2^-24 is half an fp32 step, r = 2^-8 half a bf16 step (1.0 relative).  A logit is a sum of H products (fp32 operands: of six
products of their planes, dropping less than 2^-24 of the product) formed 16 at a time in the matrix cores, so it is off by at most
    dx = (6 H / 16 + 20) u S,    S = max over rows and outputs of sum |z w| + |b|,
plus r^2 S where z = e + p is kept in two bf16 planes.  A row's sum of V1 exponentials is formed per block and then over the blocks (each addition
u relative, fewer than V1 of them in a row), each exponential off by dx and 2 u |argument|; the logarithm of it is off by
    dn = dx + (V1 + 40) u + 4 u |norm|,
so a log probability by dx + dn =: dl, and a probability relatively by about as much.  Numbers below 2^-126 count as zero: an exponential, its product
with the row's scale s and each product of planes may lose as much, so a logit's gradient (2 + s) 2^-126 and a sum of n products 6 n 2^-126
beside what its factors lose.
"""
from __future__ import annotations

import math

import numpy as np
import torch

U32, R16, TINY = 2.0 ** -24, 2.0 ** -8, 2.0 ** -126


class Layer:
    """w, b of an output layer in fp64 and the bounds that go with rows z (fp64) in type `dtype`."""

    def __init__(self, z, w, b, dtype, two_planes=False, tau=1.0):
        self.z, self.w, self.dtype = z.double(), w.double(), dtype
        b = torch.zeros(w.shape[0], dtype=torch.float64, device=w.device) if b is None else b.double()
        self.x = (self.z @ self.w.t() + b) / tau
        self.norm = torch.logsumexp(self.x, dim=1, keepdim=True)
        finite = torch.where(torch.isfinite(b), b, 0.0)
        size = float((self.z.abs() @ self.w.abs().t() + finite.abs()).max()) if self.z.numel() else 0.0
        H, V1 = w.shape[1], w.shape[0]
        self.dx = ((6 * H / 16 + 20) * U32 + (R16 * R16 if two_planes else 0.0)) * size / tau
        top = float(self.norm.abs().max()) if self.z.numel() else 0.0
        self.dl = 2 * self.dx + (V1 + 40) * U32 + 6 * U32 * max(top, 20.0)
        self.round = R16 if dtype == torch.bfloat16 else 0.0

    def gradients(self, d, rel, z_rounded=False):
        """(value, bound) of dz, dw and db for the gradient d of the logits, whose values are off by `rel` relative to their parts |d| + s p
        (`d` given as (value, size of its parts))."""
        d, size = d
        n, V1, H = d.shape[0], d.shape[1], self.w.shape[1]
        own = self.round                                    # dx is rounded to the operands' type (fp32: 2^-24, in `sums`)
        sums = (6 * max(n, V1) / 16 + 40) * U32
        scale = float(size.max()) if size.numel() else 0.0
        err = size * rel + d.abs() * own + (2 + scale) * TINY
        dz, dw, db = d @ self.w, d.t() @ self.z, d.sum(0)
        extra = own if z_rounded else 0.0                   # z in one plane
        return [(dz, err @ self.w.abs() + sums * (d.abs() @ self.w.abs()) + own * dz.abs() + 6 * V1 * TINY),
                (dw, err.t() @ self.z.abs() + (sums + extra) * (d.abs().t() @ self.z.abs()) + own * dw.abs() + 6 * n * TINY),
                (db, (size * rel).sum(0) + (n + 40) * U32 * d.abs().sum(0) + n * (2 + scale) * TINY)]


def close(got, want, bound, what):
    """got within bound of want, elementwise, NaN and infinities in the same places."""
    got, want = got.double().to(want.device), want.double()
    bound = bound if torch.is_tensor(bound) else torch.full_like(want, bound)
    fine = torch.isfinite(want)
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what
    off = (got - want).abs()[fine] - bound[fine]
    assert not off.numel() or float(off.max()) <= 0, f"{what}: {float((got - want).abs()[fine].max()):.3g} off, {float(off.max()):.3g} over the bound"


def row_loss(h, w, b, labels, logits=None, tau=1.0, weights=None):
    """Label loss (labels [N]) or distillation (labels, logits [N, K]): {name: (value, bound)}; h's rows that are left out may hold anything."""
    V1, N = w.shape[0], h.shape[0]
    lab = labels.long() if labels.dim() == 2 else labels.long()[:, None]
    there = lab >= 0
    if logits is not None:
        there &= logits != -math.inf
    wrong = (lab >= V1).any(1)
    kept = there.any(1) & ~wrong
    q = torch.zeros((N, V1), dtype=torch.float64, device=h.device)
    loss = torch.zeros(N, dtype=torch.float64, device=h.device)
    z = torch.where(kept[:, None], h.double(), 0.0)
    layer = Layer(z, w, b, h.dtype, tau=tau)
    if logits is None:
        share = there.double()
        log_q = torch.zeros_like(share)
    else:
        t = torch.where(there, logits.double() / tau, -math.inf)
        t[~kept] = 0.0
        log_q = t - torch.logsumexp(t, 1, keepdim=True)
        share = log_q.exp() * there
    at = lab.clamp(0, V1 - 1)
    terms = share * (torch.where(share > 0, log_q, 0.0) - layer.x.gather(1, at) + layer.norm)
    loss = torch.where(kept, tau * tau * torch.where(share > 0, terms, 0.0).sum(1), 0.0)
    loss[wrong] = math.nan
    q.scatter_add_(1, at, torch.where(kept[:, None], share, 0.0))
    wt = torch.ones(N, dtype=torch.float64, device=h.device) if weights is None else weights.double()
    s = torch.where(kept, tau * wt, 0.0)[:, None]
    p = (layer.x - layer.norm).exp()
    K = lab.shape[1]
    rel_q = (K + 40) * U32 * (1 if logits is None else 1 + float(logits[there].abs().nan_to_num(0, 0, 0).max() if there.any() else 0) / tau)
    bound = tau * tau * (layer.dl + rel_q * (1 + terms.abs().sum(1))) + 8 * U32 * loss.abs().nan_to_num()
    rel = layer.dl + rel_q + 8 * U32
    g = layer.gradients((s * (p - q), s.abs() * (p + q)), rel)
    return {"loss": (loss, bound), "h": g[0], "w": g[1], "b": g[2]}


def lattice(blank, emit):
    """log alpha, log beta [T + 1, U + 1] of one lattice of log probabilities (fp64 numpy), cell by cell."""
    T, U1 = blank.shape
    alpha, beta = np.full((T + 1, U1), -np.inf), np.full((T + 1, U1), -np.inf)
    for t in range(T):
        for u in range(U1):
            a = 0.0 if t == 0 and u == 0 else -np.inf
            if t:
                a = np.logaddexp(a, alpha[t - 1, u] + blank[t - 1, u])
            if u:
                a = np.logaddexp(a, alpha[t, u - 1] + emit[t, u - 1])
            alpha[t, u] = a
    beta[T, U1 - 1] = 0.0
    for t in range(T - 1, -1, -1):
        for u in range(U1 - 1, -1, -1):
            v = beta[t + 1, u] + blank[t, u]
            if u + 1 < U1:
                v = np.logaddexp(v, beta[t, u + 1] + emit[t, u])
            beta[t, u] = v
    return alpha, beta


def transducer_loss(e, p, w, b, labels, frames, counts, weights=None):
    """{name: (value, bound)} of the transducer loss."""
    B, T, H = e.shape
    U1, V1, dev = p.shape[1], w.shape[0], e.device
    loss, bound = torch.zeros(B, dtype=torch.float64), torch.zeros(B, dtype=torch.float64)
    out = {"e": [torch.zeros(e.shape, dtype=torch.float64, device=dev) for _ in range(2)], "p": [torch.zeros(p.shape, dtype=torch.float64, device=dev) for _ in range(2)],
           "w": [torch.zeros(w.shape, dtype=torch.float64, device=dev) for _ in range(2)], "b": [torch.zeros(V1, dtype=torch.float64, device=dev) for _ in range(2)]}
    for i in range(B):
        Ti, Ui = max(0, min(T, int(frames[i]))), max(0, min(U1 - 1, int(counts[i])))
        y = labels[i, :Ui].long()
        if Ti == 0:
            continue
        if bool(((y < 0) | (y >= V1 - 1)).any()):
            loss[i] = math.nan
            continue
        z = (e[i, :Ti, None].double() + p[i, None, :Ui + 1].double()).clamp(min=0).reshape(-1, H)
        layer = Layer(z, w, b, e.dtype, two_planes=e.dtype == torch.bfloat16)
        lp = (layer.x - layer.norm).reshape(Ti, Ui + 1, V1)
        blank = lp[:, :, -1].cpu().numpy()
        emit = np.full((Ti, Ui + 1), -np.inf)
        for u in range(Ui):
            emit[:, u] = lp[:, u, int(y[u])].cpu().numpy()
        alpha, beta = lattice(blank, emit)
        loss[i] = -beta[0, 0]
        arcs = Ti + Ui                          # arcs of a path; cells round two products and a sum per arc
        off = arcs * (layer.dl + 8 * U32)
        bound[i] = off + 8 * U32 * abs(float(loss[i])) if np.isfinite(beta[0, 0]) else 0.0
        if not np.isfinite(beta[0, 0]):
            continue
        wt = 1.0 if weights is None else float(weights[i])
        with np.errstate(invalid="ignore"):
            by_blank = wt * np.exp(alpha[:Ti] + blank + beta[1:] - beta[0, 0])
            after = np.concatenate([beta[:Ti, 1:], np.full((Ti, 1), -np.inf)], 1)
            by_label = wt * np.exp(alpha[:Ti] + emit + after - beta[0, 0])
        by_blank, by_label = (torch.from_numpy(np.nan_to_num(a)).to(dev) for a in (by_blank, by_label))
        pr = lp.exp()
        d = pr * (by_blank + by_label)[:, :, None]
        size = d.abs()
        d[:, :, -1] -= by_blank
        size[:, :, -1] += by_blank.abs()
        for u in range(Ui):
            d[:, u, int(y[u])] -= by_label[:, u]
            size[:, u, int(y[u])] += by_label[:, u].abs()
        rel = 3 * off + layer.dl + 40 * U32
        g = layer.gradients((d.reshape(-1, V1), size.reshape(-1, V1)), rel, z_rounded=True)
        live = (z > 0).double()
        fold = 1 + (Ti + Ui) * U32
        for k in range(2):
            # dz is kept in fp32, its sums over labels and frames are rounded once: the rounding of single rows is not part of the bound, that of sums below
            dz = (g[0][k] * live).reshape(Ti, Ui + 1, H)
            out["e"][k][i, :Ti] = dz.sum(1) * (fold if k else 1)
            out["p"][k][i, :Ui + 1] = dz.sum(0) * (fold if k else 1)
            out["w"][k] += g[1][k]
            out["b"][k] += g[2][k]
    res = {"loss": (loss, bound)}
    r = R16 if e.dtype == torch.bfloat16 else U32
    for name, (v, err) in out.items():
        res[name] = (v, err + (r * v.abs() if name != "b" else 0.0) + 64 * U32 * err)
    return res
