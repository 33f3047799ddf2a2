"""Float64 reference of cross entropy and distillation at the most features or tokens a
call takes and over the largest vocabularies, with bounds on the norms of what may be off.  There the element-wise bounds
of train_ref.py, which let every rounding err one way, are larger than the values.  The
roundings of a long sum of n terms are independent of each other: together they are a
random walk, sqrt(n) of them and not n.

MARGIN is how many standard deviations of such a walk a bound allows (each rounding is
taken at its largest, a half step, where its standard deviation is 0.58 of that)."""
import math

import torch

from tests.train_ref import HALF_STEP, targets

MARGIN = 4.0
E24 = 2.0 ** -24                 # half a step of float32


def norm(a):
    return float(a.double().norm())


def spectral(a):
    """The largest singular value, from the smaller Gram matrix."""
    g = a @ a.t() if a.shape[0] <= a.shape[1] else a.t() @ a
    return math.sqrt(float(torch.linalg.eigvalsh(g)[-1]))


class Limits:
    """Reference values, and bounds: of lse and loss element by element, of dX and dW on
    the norm of the difference."""

    def __init__(self, X, W, weight, two_terms, labels=None, index=None, logits=None, t=1.0):
        x, w = X.double(), W.double()
        N, K = x.shape
        V = w.shape[0]
        self.dtype, h = X.dtype, HALF_STEP[X.dtype]
        s = x @ w.t() / t
        # a logit: a walk over its K products, whose partial sums reach a few of the root
        # of the sum of their squares beside the logit itself; and the division by t
        top = (s.abs() + MARGIN * (x.square() @ w.square().t()).sqrt() / t)
        ds = MARGIN * math.sqrt(K + 4) * E24 * top
        self.lse = torch.logsumexp(s, 1, keepdim=True)
        q = torch.exp(s - self.lse)
        # exp of differences, a sum of V of them, log; rounded: the parts' maxima and lse
        small = 8 * E24 * (1 + s.abs().amax(1, keepdim=True) + self.lse.abs())
        dlse = (q * ds).sum(1, keepdim=True) + MARGIN * math.sqrt(V) * E24 + 2 * small
        self.dlse = dlse[:, 0]
        cols, p, logp = targets(labels, index, logits, t, V)
        live = (p != 0).any(1)
        at = s.gather(1, cols)
        self.loss = t * t * (p * (logp - at + self.lse)).sum(1)
        self.dloss = t * t * (p * (ds.gather(1, cols) + dlse + small + 16 * E24 * (1 + logp.abs()))).sum(1)
        self.lse = self.lse[:, 0]
        coef = torch.where(live, weight.double() * t, 0.0)[:, None]
        target = torch.zeros_like(q).scatter_add(1, cols, p)
        self.G = G = torch.where(live[:, None], coef * (q - target), 0.0)
        # what is off by the logits and by p's own roundings, and G's rounding
        dG = coef.abs() * (q * (ds + dlse + small) + 16 * E24 * target)
        step = (h * h if two_terms else h) if self.dtype == torch.bfloat16 else 0.0
        x = torch.where(live[:, None], x, 0.0)
        self.x, self.w, self.h = x, w, h
        self.dX, self.dW = G @ w, G.t() @ x
        gg = G.square()
        rx, rw = (gg @ w.square()).sqrt(), (gg.t() @ x.square()).sqrt()
        # G's roundings are independent: of each result, a walk over the terms of its sum.
        # The sums' own: sqrt(n) roundings of partial sums.  dX of several pieces of the
        # vocabulary adds no more of them.
        live_n = max(int(live.sum()), 1)
        self.bX = norm(dG) * spectral(w) + MARGIN * step * norm(rx) \
            + MARGIN * math.sqrt(V + 4) * E24 * (norm(self.dX) + MARGIN * norm(rx)) + h * norm(self.dX)
        self.bW = norm(dG) * spectral(x) + MARGIN * step * norm(rw) \
            + MARGIN * math.sqrt(2 * live_n + 4) * E24 * (norm(self.dW) + MARGIN * norm(rw)) + h * norm(self.dW)

    def check(self, got, ref, bound, what):
        d = (got.double() - ref)
        assert bool(d.isfinite().all()), what
        off = norm(d)
        assert off <= bound, (what, off, bound, norm(ref))

    def wrong_results_fail(self, which=("dX", "dW")):
        """Zeros, and the gradients of half of the tokens, half of the vocabulary or half
        of the features, are further off than the bounds; so are losses of 0."""
        N, V = self.G.shape
        half = self.G.clone()
        half[: (N + 1) // 2] = 0.0
        cut = self.G.clone()
        cut[:, : (V + 1) // 2] = 0.0
        for name, ref, bound, others in (
                ("dX", self.dX, self.bX, (half @ self.w, cut @ self.w)),
                ("dW", self.dW, self.bW, (half.t() @ self.x, cut.t() @ self.x))):
            if name not in which:
                continue
            assert norm(ref) > 2 * bound, (name, norm(ref), bound)
            less = ref.clone()
            less[:, : ref.shape[1] // 2] = 0.0
            for other in (*others, less):
                assert norm(other - ref) > bound, (name, norm(other - ref), bound)
        for name, ref, bound in (("lse", self.lse, self.dlse), ("loss", self.loss, self.dloss)):
            assert norm(ref) > 20 * norm(bound), (name, norm(ref), norm(bound))
