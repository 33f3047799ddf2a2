"""How far the gradients of tokens that weigh differently are off, in norm.

A value rounded to bfloat16 is off by at most half a step, h = 2^-8 of it, and evenly
within that: by h / sqrt(3) in the mean square.  The results are rounded so.  Up to 128
tokens, nothing else is; of more, the logits' gradient G is rounded before the products:
with weights that are independent of each other its roundings are, too, and add as much
again at most, sqrt(2 / 3) h together.  Weights that many tokens share (a mean over each
sequence) share their rounding of up to h: sqrt(4 / 3) h.  float32 sums are far below."""
import math

import pytest
import torch

from tests import train_ref as R
from tests.gpu_util import need_gpu
from tests.test_gpu_loss import _head, _labels, _teacher

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
H = R.HALF_STEP[BF16]


@pytest.fixture(scope="module")
def E():
    need_gpu()
    import paper_2410_05437_amd as e
    return e


def _weights(N, how, g):
    if how == "own":
        return (torch.rand(N, generator=g, device="cuda") + 0.1) / N
    # the mean over each of eight sequences of unlike lengths
    ends = torch.rand(8, generator=g, device="cuda").sort().values
    of = torch.searchsorted(ends, torch.arange(N, device="cuda") / N)
    return (1.0 / torch.bincount(of, minlength=9).clamp(min=1).float())[of] / 8


@pytest.mark.parametrize("T", [0, 16])
@pytest.mark.parametrize("how", ["own", "shared"])
@pytest.mark.parametrize("size", [(100, 520, 4000), (128, 256, 9000), (131, 520, 4000), (700, 1032, 12345), (2048, 512, 4000)],
                         ids=lambda s: "N%d_K%d_V%d" % s)
def test_weights(E, size, how, T):
    N, K, V = size
    X, W, g = _head(N, K, V, BF16, seed=51)
    w = _weights(N, how, g)
    if T:
        index, logits = _teacher(N, V, T, g)
        loss, lse, picked = E.espace_linear_distillation(X, W, index, logits, 2.0)
        dX, dW = E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, 2.0)
        ref = R.Loss(X, W, index=index, logits=logits, t=2.0)
    else:
        labels = _labels(N, V, g)
        loss, lse = E.espace_linear_cross_entropy(X, W, labels)
        dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
        ref = R.Loss(X, W, labels=labels)
    limit = H * math.sqrt(1 / 3 if N <= 128 else (2 / 3 if how == "own" else 4 / 3))
    rX, _, rW, _ = ref.grads(w, N <= 128)
    for name, got, want in (("dX", dX, rX), ("dW", dW, rW)):
        off = float((got.double() - want).norm() / want.norm())
        assert off <= limit, (name, off, limit)
