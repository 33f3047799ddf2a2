"""Float64 references of the losses and the embedding, with element-wise bounds on
what the library's arithmetic may be off (tests of espace_train.h)."""
import math

import torch

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -23       # two half steps of float32: an operation on operands rounded once


def padded(t, dtype, extra=0):
    """The matrix on rows padded to the library's alignment (and `extra` elements
    more), NaN in the padding."""
    rows, cols = t.shape
    a = 8 if dtype == torch.bfloat16 else 4
    ld = max((cols + a - 1) // a * a, a) + extra
    full = torch.full((rows, ld), float("nan"), dtype=dtype, device=t.device)
    full[:, :cols] = t
    return full[:, :cols]


def out(rows, cols, dtype, device, extra=0):
    """An output whose every element, padding included, is NaN."""
    return padded(torch.full((rows, cols), float("nan"), device=device), dtype, extra)


def padding_untouched(t):
    ld = t.stride(0)
    return bool(t.as_strided((t.shape[0], ld), (ld, 1), t.storage_offset())[:, t.shape[1]:].isnan().all())


def targets(labels=None, index=None, logits=None, t=1.0, V=None):
    """(columns [N][T], probabilities, their logarithms), float64; no entry: column
    0 and probability 0."""
    if labels is not None:
        there = (labels >= 0)[:, None]
        return labels.clamp(min=0)[:, None], there.double(), torch.zeros_like(there, dtype=torch.float64)
    there = (index >= 0) & (logits != -math.inf)
    z = torch.where(there, logits.double() / t, -math.inf)
    z = z - torch.where(there.any(1, keepdim=True), z.amax(1, keepdim=True), 0.0)
    total = torch.exp(z).sum(1, keepdim=True)
    p = torch.where(there, torch.exp(z) / total.clamp(min=1e-300), 0.0)
    return index.clamp(min=0), p, torch.where(there, z - torch.log(total.clamp(min=1e-300)), 0.0)


class Loss:
    """loss, lse, picked, and G; with bounds of the forward pass."""

    def __init__(self, X, W, labels=None, index=None, logits=None, t=1.0):
        x, w = X.double(), W.double()
        K, V = x.shape[1], w.shape[0]
        self.x, self.w, self.t, self.dtype = x, w, t, X.dtype
        s = x @ w.t() / t
        # a sum of K products, each rounded (bf16: exact), and the division by t
        ds = (K + 20) * U * (x.abs() @ w.abs().t()) / t + 4 * U * s.abs()
        self.s, self.ds = s, ds
        m = s.amax(1, keepdim=True)
        self.lse = torch.logsumexp(s, 1, keepdim=True)
        q = torch.exp(s - self.lse)
        # exp of a rounded difference, sums of at most 40 terms a level over 4 levels, log
        rel = (q * (ds + 2 * U * ((s - m).abs() + 1))).sum(1, keepdim=True)
        self.dlse = rel + (160 + V / 4096) * U + 2 * U * self.lse.abs() + 2 * U * m.abs()
        cols, p, logp = targets(labels, index, logits, t, V)
        self.cols, self.p, self.logp = cols, p, logp
        at = s.gather(1, cols)
        term = logp - at + self.lse
        z = (logp.abs() + 1) * 8 * U     # p and log p of rounded differences, and their sum of T
        self.loss = t * t * (p * term).sum(1)
        self.dloss = 1.01 * t * t * (p * (ds.gather(1, cols) + self.dlse + z + 2 * U * (logp.abs() + at.abs() + self.lse.abs()))
                                     + p * term.abs() * (z + (p.shape[1] + 20) * U)).sum(1)
        there = index >= 0 if index is not None else None
        self.picked = None if there is None else torch.where(there, at, 0.0)
        self.dpicked = None if there is None else ds.gather(1, cols)
        self.q, self.dz = q, z

    def grads(self, weight, two_terms):
        """(dX, its bound, dW, its bound) for the upstream gradient `weight`."""
        t, q = self.t, self.q
        live = (self.p != 0).any(1)
        coef = torch.where(live, weight.double() * t, 0.0)[:, None]
        target = torch.zeros_like(q).scatter_add(1, self.cols, self.p)
        dtarget = torch.zeros_like(q).scatter_add(1, self.cols, self.p * self.dz)
        G = coef * (q - target)
        G = torch.where(live[:, None], G, 0.0)
        # q of a rounded difference; G = r·c, rounded to the product's type; float32
        # sums over V or N; the output rounded
        dq = q * (self.ds + self.dlse + 4 * U * ((self.s - self.lse).abs() + 1)) + dtarget + 2 * U * (q + target)
        h = HALF_STEP[self.dtype]
        step = (h * h if two_terms else h) if self.dtype == torch.bfloat16 else 0.0
        dG = coef.abs() * dq * (1 + 2 * h) + (step + 4 * U) * G.abs() + 1e-36
        x = torch.where(live[:, None], self.x, 0.0)
        N, V = G.shape
        dX, dW = G @ self.w, G.t() @ x
        bX = 1.01 * (dG @ self.w.abs() + (V + 40) * U * (G.abs() @ self.w.abs())) * (1 + h) + h * dX.abs() + 1e-36
        bW = 1.01 * (dG.t() @ x.abs() + (2 * N + 40) * U * (G.abs().t() @ x.abs())) * (1 + h) + h * dW.abs() + 1e-36
        return dX, bX, dW, bW


def within(got, ref, bound, what):
    d = (got.double() - ref).abs()
    bad = ~(d <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), float((d / bound.clamp(min=1e-300)).max()))


def embedding_grad(tokens, dX, V, scale, start=None):
    """(dE, its bound): a float32 sum of each entry's rows, scaled, rounded."""
    x = dX.double()
    ok = (tokens >= 0) & (tokens < V)
    at = tokens[ok]
    dE = torch.zeros((V, x.shape[1]), dtype=torch.float64, device=x.device).index_add_(0, at, x[ok]) * scale
    mag = torch.zeros_like(dE).index_add_(0, at, x[ok].abs()) * abs(scale)
    n = torch.zeros(V, dtype=torch.float64, device=x.device).index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    if start is not None:
        dE, mag = dE + start.double(), mag + start.double().abs()
    return dE, 1.01 * (n[:, None] + 4) * 2.0 ** -24 * mag + HALF_STEP[dX.dtype] * 1.01 * dE.abs() + 1e-40
