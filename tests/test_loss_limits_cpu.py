"""The bounds of tests/loss_limits_ref.py tell right results from wrong ones."""
import pytest
import torch

from tests import train_ref as R
from tests.loss_limits_ref import Limits

BF16, F32 = torch.bfloat16, torch.float32


def _inputs(N, K, V, dtype, T):
    g = torch.Generator().manual_seed(N + K + V)
    X = torch.randn(N, K, generator=g) * torch.exp(0.3 * torch.randn(1, K, generator=g))
    W = torch.randn(V, K, generator=g) * (2.0 * K ** -0.5)
    w = torch.rand(N, generator=g) / N
    if T:
        target = dict(index=torch.randint(0, V, (N, T), generator=g), logits=torch.randn(N, T, generator=g) * 3.0, t=2.0)
    else:
        labels = torch.randint(0, V, (N,), generator=g)
        labels[torch.rand(N, generator=g) < 0.2] = -100
        labels[0], labels[1] = V - 1, 0
        target = dict(labels=labels)
    return X.to(dtype), W.to(dtype), w, target


@pytest.mark.parametrize("T", [0, 3])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(3, 1 << 21, 40), (140, 1 << 18, 40), ((1 << 18) - 1, 16, 130)],
                         ids=lambda s: "N%d_K%d_V%d" % s)
def test_bounds(size, dtype, T):
    N, K, V = size
    X, W, w, target = _inputs(N, K, V, dtype, T)
    two = N <= 128
    ref = Limits(X, W, w, two, **target)
    ref.wrong_results_fail()
    # the plain form in float32 is within them, with G rounded as the library rounds it
    t = target.get("t", 1.0)
    x, m = X.float(), W.float()
    s = x @ m.t() / t
    lse = torch.logsumexp(s, 1)
    cols, p, logp = R.targets(target.get("labels"), target.get("index"), target.get("logits"), t, V)
    p, logp = p.float(), logp.float()
    loss = t * t * (p * (logp - s.gather(1, cols) + lse[:, None])).sum(1)
    G = torch.exp(s - lse[:, None]).scatter_add(1, cols, -p) * (t * w[:, None])
    G = torch.where((p != 0).any(1)[:, None], G, 0.0)
    if dtype == BF16:
        c = G.abs().max()
        G = (G / c).bfloat16().float() * c + (((G / c) - (G / c).bfloat16().float()).bfloat16().float() * c if two else 0.0)
    R.within(lse, ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    ref.check((G @ m).to(dtype), ref.dX, ref.bX, "dX")
    ref.check((G.t() @ x).to(dtype), ref.dW, ref.bW, "dW")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_bounds_over_large_vocabularies(dtype):
    X, W, w, target = _inputs(2, 8, (1 << 22) + 5, dtype, 0)
    ref = Limits(X, W, w, True, **target)
    ref.wrong_results_fail(which=("dX",))
