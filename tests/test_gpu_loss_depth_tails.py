"""The losses' tiled products where a depth ends inside the tiles' last step of 64: the
features of the logits, the vocabulary of dX, the tokens with a target of dW.  A depth of
32 more than whole steps leaves the step's second half wholly past the end; two steps
leave no others between the first loads and that half."""
import pytest
import torch

from tests import train_ref as R
from tests.gpu_util import need_gpu
from tests.test_gpu_loss import _fused, _head, _teacher, _weight

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def E():
    need_gpu()
    import paper_2410_05437_amd as e
    return e


# tokens, those with a target, features, vocabulary
ENDS = [(700, 608, 1056, 12320), (700, 607, 1055, 12319), (700, 609, 1057, 12321), (700, 616, 1064, 12328),
        (700, 577, 1025, 12289), (700, 639, 1087, 12351), (4500, 96, 96, 9056), (4500, 95, 95, 9120),
        (4500, 32, 97, 9057), (4500, 4448, 72, 9025), (1300, 160, 160, 40032)]


@pytest.mark.parametrize("T", [0, 3])
@pytest.mark.parametrize("size", ENDS, ids=lambda s: "N%d_live%d_K%d_V%d" % s)
def test_depths_that_end_inside_a_step(E, capfd, size, T):
    N, live, K, V = size
    t = 2.0 if T else 1.0
    X, W, g = _head(N, K, V, BF16, seed=21)
    on = torch.zeros(N, dtype=torch.bool, device="cuda")
    on[torch.randperm(N, generator=g, device="cuda")[:live]] = True
    w = _weight(N, g)
    dX, dW = R.out(N, K, BF16, "cuda"), R.out(V, K, BF16, "cuda")
    if T:
        index, logits = _teacher(N, V, T, g)
        index[~on] = -1
        (loss, lse, picked), f1 = _fused(capfd, lambda: E.espace_linear_distillation(X, W, index, logits, t))
        _, f2 = _fused(capfd, lambda: E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t, dX=dX, dW=dW))
        ref = R.Loss(X, W, index=index, logits=logits, t=t)
    else:
        labels = torch.where(on, torch.randint(0, V, (N,), generator=g, device="cuda"), -1)
        (loss, lse), f1 = _fused(capfd, lambda: E.espace_linear_cross_entropy(X, W, labels))
        _, f2 = _fused(capfd, lambda: E.espace_linear_cross_entropy_backward(w, X, W, labels, lse, dX=dX, dW=dW))
        ref = R.Loss(X, W, labels=labels)
    assert f1 == [True] and f2 == [True]
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    rX, bX, rW, bW = ref.grads(w, False)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")
    assert not dX[~on].any()
