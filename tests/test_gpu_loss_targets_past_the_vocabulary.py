"""How far a target past the vocabulary reaches: which losses and gradients are NaN, and
that the others are those of a call without it."""
import pytest
import torch

from tests import train_ref as R
from tests.gpu_util import need_gpu
from tests.test_gpu_loss import _head, _labels, _weight

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def E():
    need_gpu()
    import paper_2410_05437_amd as e
    return e


CASES = pytest.mark.parametrize("dtype,size", [(BF16, (4, 72, 700)), (BF16, (300, 72, 5000)), (BF16, (700, 1032, 12345)),
                                               (BF16, (2100, 136, 1300)), (F32, (4, 72, 700)), (F32, (300, 72, 5000))],
                                ids=lambda s: "N%d_K%d_V%d" % s if isinstance(s, tuple) else str(s).split(".")[-1])


@CASES
@pytest.mark.parametrize("past", [0, 1 << 40])
def test_a_label(E, dtype, size, past):
    N, K, V = size
    X, W, g = _head(N, K, V, dtype, seed=31)
    labels, w = _labels(N, V, g, none=0.0), _weight(N, g)
    ref = R.Loss(X, W, labels=labels)
    rX, bX, _, _ = ref.grads(w, N <= 128)
    labels[3] = V + past
    other = torch.arange(N, device="cuda") != 3
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss[other], ref.loss[other], ref.dloss[other], "loss")
    R.within(dX[other], rX[other], bX[other], "dX")
    assert bool(loss[3].isnan()) and bool(dX[3].isnan().all()) and bool(dW.isnan().all())


@CASES
@pytest.mark.parametrize("T", [2, 70])
def test_a_teachers_entry(E, dtype, size, T):
    N, K, V = size
    t = 2.0
    X, W, g = _head(N, K, V, dtype, seed=32)
    index = torch.randint(0, V, (N, T), generator=g, device="cuda")
    logits, w = torch.randn(N, T, generator=g, device="cuda"), _weight(N, g)
    index[3, 0], index[3, 1] = V - 1, 5
    ref = R.Loss(X, W, index=index, logits=logits, t=t)
    rX, bX, rW, bW = ref.grads(w, N <= 128)
    hit = torch.zeros(V, dtype=torch.bool, device="cuda")
    hit[index[3]] = True
    index[3, 0] = V + 11
    other = torch.arange(N, device="cuda") != 3
    loss, lse, picked = E.espace_linear_distillation(X, W, index, logits, t)
    dX, dW = E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss[other], ref.loss[other], ref.dloss[other], "loss")
    R.within(dX[other], rX[other], bX[other], "dX")
    R.within(dW[~hit], rW[~hit], bW[~hit], "dW")
    assert bool(loss[3].isnan()) and bool(dX[3].isnan().all()) and bool(dW[hit].isnan().all())
    # of no weight: no gradient
    w[3] = 0.0
    rX, bX, rW, bW = ref.grads(w, N <= 128)
    dX, dW = E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")
