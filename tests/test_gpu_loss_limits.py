"""The losses at the most features and the most tokens that a call takes, and over large
vocabularies, against float64 with bounds that hold there (tests/loss_limits_ref.py)."""
import pytest
import torch

from tests import train_ref as R
from tests.gpu_util import need_gpu
from tests.loss_limits_ref import Limits
from tests.test_gpu_loss import _head, _labels, _weight

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
MOST = 1 << 21


@pytest.fixture(scope="module")
def E():
    need_gpu()
    import paper_2410_05437_amd as e
    return e


@pytest.mark.parametrize("T", [0, 3])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(3, MOST, 40), (140, MOST, 40), (MOST - 1, 16, 130)], ids=lambda s: "N%d_K%d_V%d" % s)
def test_limits(E, size, dtype, T):
    N, K, V = size
    X, W, g = _head(N, K, V, dtype, seed=41)
    w = _weight(N, g)
    dX, dW = R.out(N, K, dtype, "cuda"), R.out(V, K, dtype, "cuda")
    if T:
        t = 2.0
        index = torch.randint(0, V, (N, T), generator=g, device="cuda")
        logits = torch.randn(N, T, generator=g, device="cuda") * 3.0
        ref = Limits(X, W, w, N <= 128, index=index, logits=logits, t=t)
        loss, lse, picked = E.espace_linear_distillation(X, W, index, logits, t)
        E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t, dX=dX, dW=dW)
    else:
        labels = _labels(N, V, g)
        ref = Limits(X, W, w, N <= 128, labels=labels)
        loss, lse = E.espace_linear_cross_entropy(X, W, labels)
        E.espace_linear_cross_entropy_backward(w, X, W, labels, lse, dX=dX, dW=dW)
    ref.wrong_results_fail()
    R.within(lse, ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    ref.check(dX, ref.dX, ref.bX, "dX")
    ref.check(dW, ref.dW, ref.bW, "dW")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 8, (1 << 25) + 5), (2, 8, (1 << 25) + 5), (40, 40, 1500001), (300, 40, 400003)],
                         ids=lambda s: "N%d_K%d_V%d" % s)
def test_gradient_of_the_activations_over_large_vocabularies(E, size, dtype):
    """(dW's rows have a term a token: the element-wise bounds hold them.)"""
    N, K, V = size
    X, W, g = _head(N, K, V, dtype, seed=42)
    labels, w = torch.randint(0, V, (N,), generator=g, device="cuda"), _weight(N, g)
    ref = Limits(X, W, w, N <= 128, labels=labels)
    ref.wrong_results_fail(which=("dX",))
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    dX, _ = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse, want_dw=False)
    R.within(lse, ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    ref.check(dX, ref.dX, ref.bX, "dX")
