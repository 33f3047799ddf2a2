"""Cross entropy and distillation through a linear head, forward and backward, against
float64 (tests/train_ref.py)."""
import math

import pytest
import torch

from tests import train_ref as R
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def E():
    need_gpu()
    import paper_2410_05437_amd as e
    return e


def _head(N, K, V, dtype, seed=0, spread=2.0, extra=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + N + K + V)
    X = torch.randn(N, K, generator=g, device="cuda") * torch.exp(0.3 * torch.randn(1, K, generator=g, device="cuda"))
    W = torch.randn(V, K, generator=g, device="cuda") * spread * K ** -0.5
    return R.padded(X.to(dtype), dtype, extra), R.padded(W.to(dtype), dtype, extra), g


def _labels(N, V, g, none=0.2):
    labels = torch.randint(0, V, (N,), generator=g, device="cuda")
    labels[torch.rand(N, generator=g, device="cuda") < none] = -100
    if N > 2:
        labels[0], labels[1] = V - 1, 0
    return labels


def _weight(N, g):
    return torch.rand(N, generator=g, device="cuda") / N


SIZES = [(1, 64, 1), (1, 8, 2), (2, 100, 1003), (3, 1000, 517), (17, 256, 4096), (33, 72, 4097), (130, 1003, 2049),
         (300, 520, 5000), (601, 1000, 5003), (1025, 264, 777), (2100, 136, 1300), (4500, 72, 9001),
         (129, 520, 3000), (700, 1032, 12345), (2051, 777, 4160), (4096, 512, 12000)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "N%d_K%d_V%d" % s)
def test_cross_entropy(E, size, dtype):
    N, K, V = size
    X, W, g = _head(N, K, V, dtype)
    labels, w = _labels(N, V, g), _weight(N, g)
    ws = torch.full((E.espace_linear_loss_workspace_bytes(False, N, K, V, 0, dtype),), 255, dtype=torch.uint8, device="cuda")
    loss, lse = E.espace_linear_cross_entropy(X, W, labels, workspace=ws)
    ref = R.Loss(X, W, labels=labels)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    assert bool((loss[labels < 0] == 0).all())
    ws = torch.full((E.espace_linear_loss_workspace_bytes(True, N, K, V, 0, dtype),), 255, dtype=torch.uint8, device="cuda")
    dX, dW = R.out(N, K, dtype, "cuda"), R.out(V, K, dtype, "cuda")
    E.espace_linear_cross_entropy_backward(w, X, W, labels, lse, dX=dX, dW=dW, workspace=ws)
    rX, bX, rW, bW = ref.grads(w, N <= 128)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")
    assert R.padding_untouched(dX) and R.padding_untouched(dW)
    assert bool((dX[labels < 0] == 0).all())
    # each gradient alone, and the calls again: the same bits
    dX1, none = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse, want_dw=False)
    assert none is None
    none, dW1 = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse, want_dx=False)
    assert none is None and torch.equal(dX, dX1) and torch.equal(dW, dW1)
    loss1, lse1 = E.espace_linear_cross_entropy(X, W, labels)
    assert torch.equal(loss, loss1) and torch.equal(lse, lse1)


def _teacher(N, V, T, g, spread=3.0):
    index = torch.stack([torch.randperm(V, generator=g, device="cuda")[:T] if V >= T else
                         torch.randint(0, V, (T,), generator=g, device="cuda") for _ in range(N)])
    logits = torch.randn(N, T, generator=g, device="cuda") * spread
    return index, logits


KD = [(1, 64, 3, 1, 1.0), (5, 100, 1000, 7, 2.0), (33, 72, 4097, 64, 1.0), (65, 256, 1003, 65, 4.0), (40, 64, 500, 200, 0.5),
      (12, 40, 70, 300, 1.0), (9, 40, 2000, 1024, 3.0), (300, 520, 3001, 32, 2.0), (2050, 136, 700, 16, 1.5),
      (4300, 72, 9001, 3, 2.0), (700, 1032, 12345, 70, 2.0), (2051, 777, 4160, 128, 1.0), (1030, 512, 9001, 1000, 3.0)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", KD, ids=lambda s: "N%d_K%d_V%d_T%d_t%g" % s)
def test_distillation(E, size, dtype):
    N, K, V, T, t = size
    X, W, g = _head(N, K, V, dtype, seed=1)
    index, logits = _teacher(N, V, T, g)
    index[torch.rand(N, T, generator=g, device="cuda") < 0.2] = -1
    w = _weight(N, g)
    if N > 4:
        index[1] = -7                               # no target
        logits[2] = -math.inf                       # the same
        logits[3, : T // 2] = -math.inf             # entries of probability 0
        index[4] = index[4].amax()                  # one entry in all places
        if T > 2:
            index[0, 2] = index[0, 0]               # one entry twice
    # rows apart by more than T
    wide = torch.full((N, T + 3), -1, device="cuda")
    wide[:, :T] = index
    index = wide[:, :T]
    ws = torch.full((E.espace_linear_loss_workspace_bytes(False, N, K, V, T, dtype),), 255, dtype=torch.uint8, device="cuda")
    picked = torch.full((N, T + 1), float("nan"), device="cuda")
    loss, lse, _ = E.espace_linear_distillation(X, W, index, logits, t, picked=picked[:, :T], workspace=ws)
    assert bool(picked[:, T:].isnan().all())
    picked = picked[:, :T]
    ref = R.Loss(X, W, index=index, logits=logits, t=t)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(picked, ref.picked, ref.dpicked, "picked")
    R.within(loss, ref.loss, ref.dloss, "loss")
    ws = torch.full((E.espace_linear_loss_workspace_bytes(True, N, K, V, T, dtype),), 255, dtype=torch.uint8, device="cuda")
    dX, dW = R.out(N, K, dtype, "cuda"), R.out(V, K, dtype, "cuda")
    E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t, dX=dX, dW=dW, workspace=ws)
    rX, bX, rW, bW = ref.grads(w, N <= 128)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")
    assert R.padding_untouched(dX) and R.padding_untouched(dW)
    dX1, _ = E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t, want_dw=False)
    _, dW1 = E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t, want_dx=False)
    assert torch.equal(dX, dX1) and torch.equal(dW, dW1)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N", [5, 300, 700])
def test_distillation_from_one_entry_is_cross_entropy(E, N, dtype):
    K, V = 264, 3001
    X, W, g = _head(N, K, V, dtype, seed=2)
    labels, w = _labels(N, V, g), _weight(N, g)
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    z = torch.randn(N, 1, generator=g, device="cuda")
    loss2, lse2, picked = E.espace_linear_distillation(X, W, labels[:, None], z)
    assert torch.equal(lse, lse2)
    R.within(loss2, loss.double(), 4 * R.U * lse.double().abs() + 4 * R.U * picked[:, 0].double().abs(), "loss")


@pytest.mark.parametrize("N", [6, 40, 300, 1200])
def test_tokens_without_a_target_add_nothing(E, N):
    """Their rows of X, their upstream gradients and the logits of their row hold NaN
    and infinities; all of the tokens without one: zeros."""
    K, V, dtype = 136, 1303, BF16
    X, W, g = _head(N, K, V, dtype, seed=3)
    labels, w = _labels(N, V, g, none=0.3), _weight(N, g)
    labels[0], labels[2], labels[4] = -1, -100, -(1 << 40)
    none = labels < 0
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
    X2, w2 = X.clone(), w.clone()
    X2[0], X2[2], X2[4, 3] = float("nan"), math.inf, -math.inf
    X2 = R.padded(X2, dtype)
    w2[0], w2[2] = float("nan"), math.inf
    loss2, lse2 = E.espace_linear_cross_entropy(X2, W, labels)
    assert torch.equal(loss, loss2) and bool((loss2[none] == 0).all())
    assert torch.equal(lse[~none], lse2[~none])
    dX2, dW2 = E.espace_linear_cross_entropy_backward(w2, X2, W, labels, lse2)
    assert torch.equal(dX, dX2) and torch.equal(dW, dW2)
    gone = torch.full_like(labels, -1)
    loss3, lse3 = E.espace_linear_cross_entropy(X2, W, gone)
    dX3, dW3 = E.espace_linear_cross_entropy_backward(w2, X2, W, gone, lse3)
    assert not loss3.any() and not dX3.any() and not dW3.any()
    index, logits = torch.stack([labels, labels], 1), torch.zeros(N, 2, device="cuda")
    loss4, lse4, picked = E.espace_linear_distillation(X2, W, index, logits)
    assert bool((loss4[none] == 0).all()) and bool(loss4[~none].isfinite().all()) and bool((picked[none] == 0).all())
    dX4, dW4 = E.espace_linear_distillation_backward(w2, X2, W, index, logits, lse4, picked)
    assert bool(dX4.isfinite().all()) and bool(dW4.isfinite().all()) and not dX4[none].any()


@pytest.mark.parametrize("N", [4, 300, 600])
def test_targets_past_the_vocabulary_give_nan(E, N):
    K, V = 72, 700
    X, W, g = _head(N, K, V, BF16, seed=4)
    labels, w = _labels(N, V, g, none=0.0), _weight(N, g)
    labels[3] = V
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
    other = torch.arange(N, device="cuda") != 3
    assert bool(loss[3].isnan()) and bool(loss[other].isfinite().all()) and bool(lse.isfinite().all())
    assert bool(dX[3].isnan().all()) and bool(dX[other].isfinite().all()) and bool(dW.isnan().any())
    index = torch.stack([labels, labels - 1], 1)
    loss, lse, picked = E.espace_linear_distillation(X, W, index, torch.zeros(N, 2, device="cuda"))
    assert bool(loss[3].isnan()) and bool(loss[other].isfinite().all())
    dX, dW = E.espace_linear_distillation_backward(w, X, W, index, torch.zeros(N, 2, device="cuda"), lse, picked)
    assert bool(dX[3].isnan().any()) and bool(dX[other].isfinite().all()) and bool(dW.isnan().any())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N", [7, 300])
def test_large_logits(E, N, dtype):
    """Logits of some hundreds: their exponentials overflow float32, and all but a
    few of the differences' underflow."""
    K, V = 64, 2003
    X, W, g = _head(N, K, V, dtype, seed=5, spread=200.0)
    labels, w = _labels(N, V, g), _weight(N, g)
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    ref = R.Loss(X, W, labels=labels)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
    rX, bX, rW, bW = ref.grads(w, N <= 128)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")


@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e25])
def test_upstream_gradients_of_any_size(E, scale):
    N, K, V = 70, 64, 500
    X, W, g = _head(N, K, V, BF16, seed=6)
    labels, w = _labels(N, V, g), torch.rand(N, generator=g, device="cuda") - 0.5
    w[5] = 0.0
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    dX, dW = E.espace_linear_cross_entropy_backward(w * scale, X, W, labels, lse)
    rX, bX, rW, bW = R.Loss(X, W, labels=labels).grads(w * scale, N <= 128)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")
    assert not dX[5].any()


def test_no_tokens(E):
    W = R.padded(torch.ones(10, 16, device="cuda").bfloat16(), BF16)
    X, labels = torch.empty((0, 16), dtype=BF16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    v = torch.empty(0, device="cuda")
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    assert loss.shape == lse.shape == (0,)
    dX, dW = E.espace_linear_cross_entropy_backward(v, X, W, labels, v, dW=R.out(10, 16, BF16, "cuda"))
    assert dX.shape == (0, 16) and not dW.any()
    i, z = torch.empty((0, 3), dtype=torch.int64, device="cuda"), torch.empty((0, 3), device="cuda")
    loss, lse, picked = E.espace_linear_distillation(X, W, i, z)
    dX, dW = E.espace_linear_distillation_backward(v, X, W, i, z, lse, picked)
    assert loss.shape == (0,) and not dW.any()


def test_gradients_against_differences(E):
    """Central differences of the library's own loss in float32 along random
    directions.  The loss's third derivative along a unit direction of X is at most
    2·max|w|³ (the third central moment of the row's logits), so the difference is off
    by h²/3·max|w|³; the two losses' rounding adds 2·dloss / 2h."""
    N, K, V, T, t, h = 3, 24, 50, 4, 2.0, 1e-2
    X, W, g = _head(N, K, V, F32, seed=7)
    labels = _labels(N, V, g, none=0.0)
    index, logits = _teacher(N, V, T, g)
    one = torch.ones(N, device="cuda")
    for kind in ("labels", "teacher"):
        def run(X, W):
            if kind == "labels":
                return E.espace_linear_cross_entropy(R.padded(X, F32), R.padded(W, F32), labels)
            return E.espace_linear_distillation(R.padded(X, F32), R.padded(W, F32), index, logits, t)
        if kind == "labels":
            _, lse = run(X, W)
            dX, dW = E.espace_linear_cross_entropy_backward(one, X, W, labels, lse)
            ref = R.Loss(X, W, labels=labels)
        else:
            _, lse, picked = run(X, W)
            dX, dW = E.espace_linear_distillation_backward(one, X, W, index, logits, lse, picked, t)
            ref = R.Loss(X, W, index=index, logits=logits, t=t)
        noise = float(ref.dloss.max()) / h * 2
        for which, grad in (("X", dX), ("W", dW)):
            d = torch.randn(grad.shape, generator=g, device="cuda")
            d = d / d.norm(dim=1, keepdim=True)
            if which == "X":
                up, down = run(X + h * d, W)[0], run(X - h * d, W)[0]
                got, m = (grad * d).sum(1), float(W.norm(dim=1).max())
            else:
                up, down = run(X, W + h * d)[0].sum()[None], run(X, W - h * d)[0].sum()[None]
                got, m = (grad * d).sum()[None], float(X.norm(dim=1).max())
            diff = (up - down) / (2 * h)
            # N losses in one sum of dW's; the direction's own rounding to float32
            tol = N * (noise + h * h / 3 * m ** 3 + 1e-5 * m)
            assert bool(((got - diff).abs() <= tol).all()), (kind, which, (got - diff).abs().max(), tol)


@pytest.mark.parametrize("N", [9, 700])
def test_captured_calls(E, N):
    """Both losses with their gradients in one captured graph, replayed between eager
    calls on other inputs that share nothing but the allocator."""
    K, V, T = 264, 1500, 5
    X, W, g = _head(N, K, V, BF16, seed=8)
    labels, w = _labels(N, V, g), _weight(N, g)
    index, logits = _teacher(N, V, T, g)
    ws = [torch.empty(E.espace_linear_loss_workspace_bytes(b, N, K, V, n, BF16), dtype=torch.uint8, device="cuda")
          for b in (False, True) for n in (0, T)]

    def run(X, w):
        loss, lse = E.espace_linear_cross_entropy(X, W, labels, workspace=ws[0])
        dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse, workspace=ws[2])
        loss2, lse2, picked = E.espace_linear_distillation(X, W, index, logits, 2.0, workspace=ws[1])
        dX2, dW2 = E.espace_linear_distillation_backward(w, X, W, index, logits, lse2, picked, 2.0, workspace=ws[3])
        return loss, lse, dX, dW, loss2, lse2, picked, dX2, dW2

    run(X, w)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run(X, w)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    Xin, win = X.clone(), w.clone()
    Xin = R.padded(Xin, BF16)
    with torch.cuda.graph(graph):
        outs = run(Xin, win)
    for k in range(4):
        Xk = (X.float() * (1 + 0.1 * k)).bfloat16()
        Xin.copy_(Xk)
        win.copy_(w * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        want = run(R.padded(Xk, BF16), w * (k + 1))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


def test_two_streams_at_once(E):
    N, K, V = 400, 264, 6000
    X, W, g = _head(N, K, V, BF16, seed=9)
    labels, w = _labels(N, V, g), _weight(N, g)
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    want = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                l, e = E.espace_linear_cross_entropy(X, W, labels)
                got.append((l, e, *E.espace_linear_cross_entropy_backward(w, X, W, labels, e)))
    torch.cuda.synchronize()
    for r in got:
        assert all(torch.equal(a, b) for a, b in zip(r, (loss, lse, *want)))


def test_a_retraining_step(E):
    """Embedding, a projected layer, the loss through a projected head, and the way
    back: every gradient against a float64 chain of the bfloat16 weights.  Rounded to
    bfloat16 on the way: X, Z, Y, Zh, the folded weights, and on the way back dZh, dY,
    the layer's two products, dX; relative errors of half a step each (2^-8 at most, a
    half of that on average), twelve of them at most one after the other."""
    N, K, M, L, V = 300, 256, 384, 96, 1500
    g = torch.Generator(device="cuda").manual_seed(77)

    def mat(r, c, s):
        return R.padded((torch.randn(r, c, generator=g, device="cuda") * s).bfloat16(), BF16)

    table, W, head = mat(V, K, 1.0), mat(M, K, K ** -0.5), mat(V, M, 2 * M ** -0.5)
    P = R.padded(torch.linalg.qr(torch.randn(K, L, generator=g, device="cuda"))[0].t().contiguous().bfloat16(), BF16)
    Ph = R.padded(torch.linalg.qr(torch.randn(M, L, generator=g, device="cuda"))[0].t().contiguous().bfloat16(), BF16)
    tokens = torch.randint(0, V, (N,), generator=g, device="cuda")
    tokens[:40] = 7
    tokens[50] = -1
    labels, w = _labels(N, V, g), torch.full((N,), 1.0 / N, device="cuda")
    X = E.espace_embedding(tokens, table, scale=1.5)
    Wf = E.espace_fold_weights(W, P)
    Z = E.espace_project(P, X)
    Y = E.espace_expand(Z, Wf)
    Hf = E.espace_fold_weights(head, Ph)
    Zh = E.espace_project(Ph, Y)
    loss, lse = E.espace_linear_cross_entropy(Zh, Hf, labels)
    dZh, dHf = E.espace_linear_cross_entropy_backward(w, Zh, Hf, labels, lse)
    # Zh = Y·Phᵀ: its gradient with the transposed projection as the weight
    dY, _ = E.espace_dense_linear_backward(dZh, Y, Ph, want_dw=False)
    dX, dW = E.espace_projected_linear_backward(dY, Z, P, Wf)
    dE = E.espace_embedding_backward(tokens, dX, V, scale=1.5)

    leaf = {n: v.double().clone().requires_grad_() for n, v in (("table", table), ("W", W), ("Hf", Hf))}
    rows = torch.cat([leaf["table"], torch.zeros(1, K, device="cuda", dtype=torch.float64)])
    x = 1.5 * rows[torch.where(tokens < 0, V, tokens)]
    y = (x @ P.double().t()) @ (leaf["W"] @ P.double().t()).t()
    s = (y @ Ph.double().t()) @ leaf["Hf"].t()
    ref = torch.nn.functional.cross_entropy(s, labels, ignore_index=-100, reduction="none")
    (ref.sum() / N).backward()
    step = 2.0 ** -8
    for name, got, want in (("loss", loss, ref.detach()), ("dHf", dHf, leaf["Hf"].grad), ("dW", dW, leaf["W"].grad),
                            ("dE", dE, leaf["table"].grad)):
        off = float((got.double() - want).norm() / want.norm())
        assert off <= 12 * step, (name, off)
    assert not dE[torch.bincount(tokens[tokens >= 0], minlength=V) == 0].any()


@pytest.mark.parametrize("T", [0, 3])
def test_leading_dimensions_past_the_tiles_offsets(E, T):
    """A head whose rows lie so far apart that it spans 2^31 elements and more."""
    N, K, V, t = 4300, 72, 9001, 2.0 if T else 1.0
    X, W, g = _head(N, K, V, BF16, seed=10)
    apart = (1 << 31) // V + 9 & ~7
    far = torch.zeros((V * apart,), dtype=BF16, device="cuda").as_strided((V, K), (apart, 1))
    far.copy_(W)
    w = _weight(N, g)
    if T:
        index, logits = _teacher(N, V, T, g)
        loss, lse, picked = E.espace_linear_distillation(X, far, index, logits, t)
        dX, dW = E.espace_linear_distillation_backward(w, X, far, index, logits, lse, picked, t)
        ref = R.Loss(X, W, index=index, logits=logits, t=t)
        R.within(picked, ref.picked, ref.dpicked, "picked")
    else:
        labels = _labels(N, V, g)
        loss, lse = E.espace_linear_cross_entropy(X, far, labels)
        dX, dW = E.espace_linear_cross_entropy_backward(w, X, far, labels, lse)
        ref = R.Loss(X, W, labels=labels)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    rX, bX, rW, bW = ref.grads(w, False)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")


def _fused(capfd, call):
    """(call(), whether each of its loss plans kept the logits in the tiles)."""
    capfd.readouterr()
    out = call()
    return out, [line.split("fused=")[1][0] == "1" for line in capfd.readouterr().err.splitlines()
                 if line.startswith("espace loss plan")]


@pytest.mark.parametrize("T", [0, 5])
@pytest.mark.parametrize("live", [0, 1, 191, 256, 257, 699, 700])
def test_few_tokens_with_a_target(E, capfd, live, T):
    """The tiles' products run over the tokens with a gradient alone."""
    N, K, V, t = 700, 1032, 12345, 2.0 if T else 1.0
    X, W, g = _head(N, K, V, BF16, seed=11)
    some = torch.randperm(N, generator=g, device="cuda")[:live]
    on = torch.zeros(N, dtype=torch.bool, device="cuda")
    on[some] = True
    X = R.padded(torch.where(on[:, None], X, float("nan")), BF16)
    w = torch.where(on, _weight(N, g), float("inf"))
    dX, dW = R.out(N, K, BF16, "cuda", extra=8), R.out(V, K, BF16, "cuda", extra=8)
    clean = torch.where(on[:, None], X, 0.0).contiguous()
    wc = torch.where(on, w, 0.0)
    if T:
        index, logits = _teacher(N, V, T, g)
        index[~on] = -1
        (loss, lse, picked), f1 = _fused(capfd, lambda: E.espace_linear_distillation(X, W, index, logits, t))
        _, f2 = _fused(capfd, lambda: E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t, dX=dX, dW=dW))
        ref = R.Loss(clean, W, index=index, logits=logits, t=t)
    else:
        labels = torch.where(on, torch.randint(0, V, (N,), generator=g, device="cuda"), -1)
        (loss, lse), f1 = _fused(capfd, lambda: E.espace_linear_cross_entropy(X, W, labels))
        _, f2 = _fused(capfd, lambda: E.espace_linear_cross_entropy_backward(w, X, W, labels, lse, dX=dX, dW=dW))
        ref = R.Loss(clean, W, labels=labels)
    assert f1 == [True] and f2 == [True]
    R.within(loss, ref.loss, ref.dloss, "loss")
    rX, bX, rW, bW = ref.grads(wc, False)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")
    assert not dX[~on].any() and R.padding_untouched(dX) and R.padding_untouched(dW)


@pytest.mark.parametrize("size", [(1, 40, 3000), (16, 1999, 700), (33, 33, 40000), (100, 250, 300), (100, 257, 2500), (450, 131, 75000),
                                  (450, 131, 65556)],
                         ids=lambda s: "N%d_K%d_V%d" % s)
@pytest.mark.parametrize("apart", [False, True], ids=["packed", "far"])
def test_float32_products_read_their_operands_as_they_lie(E, size, apart):
    """Pieces of the vocabulary whose last has few columns, tokens without a target that
    hold NaN, and a head whose rows span 2^32 bytes and more: the same gradients."""
    N, K, V = size
    X, W, g = _head(N, K, V, F32, seed=12)
    labels, w = _labels(N, V, g), _weight(N, g)
    none = labels < 0
    clean = torch.where(none[:, None], 0.0, X)
    X = R.padded(torch.where(none[:, None], float("nan"), X), F32)
    if apart:
        ld = ((1 << 30) // V + 7) & ~3
        far = torch.full((V * ld,), float("nan"), dtype=F32, device="cuda").as_strided((V, K), (ld, 1))
        far.copy_(W)
    else:
        far = W
    loss, lse = E.espace_linear_cross_entropy(X, far, labels)
    dX, dW = R.out(N, K, F32, "cuda", extra=4), R.out(V, K, F32, "cuda", extra=4)
    E.espace_linear_cross_entropy_backward(w, X, far, labels, lse, dX=dX, dW=dW)
    ref = R.Loss(clean, W, labels=labels)
    R.within(lse[~none, None], ref.lse[~none], ref.dlse[~none], "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    rX, bX, rW, bW = ref.grads(w, False)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")
    assert R.padding_untouched(dX) and R.padding_untouched(dW) and not dX[none].any()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(1, 8, (1 << 25) + 5), (2, 8, (1 << 25) + 5), (40, 40, 1500001)],
                         ids=lambda s: "N%d_K%d_V%d" % s)
def test_large_vocabularies(E, size, dtype):
    N, K, V = size
    X, W, g = _head(N, K, V, dtype, seed=13)
    labels, w = torch.randint(0, V, (N,), generator=g, device="cuda"), _weight(N, g)
    labels[0] = V - 1
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
    ref = R.Loss(X, W, labels=labels)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    rX, bX, rW, bW = ref.grads(w, N <= 128)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T", [0, 3])
def test_most_tokens_a_call_takes(E, dtype, T):
    N, K, V, t = (1 << 21) - 1, 16, 130, 2.0 if T else 1.0
    X, W, g = _head(N, K, V, dtype, seed=14)
    w = _weight(N, g)
    if T:
        index = torch.randint(0, V, (N, T), generator=g, device="cuda")
        logits = torch.randn(N, T, generator=g, device="cuda") * 3.0
        loss, lse, picked = E.espace_linear_distillation(X, W, index, logits, t)
        dX, dW = E.espace_linear_distillation_backward(w, X, W, index, logits, lse, picked, t)
        ref = R.Loss(X, W, index=index, logits=logits, t=t)
        R.within(picked, ref.picked, ref.dpicked, "picked")
    else:
        labels = _labels(N, V, g)
        loss, lse = E.espace_linear_cross_entropy(X, W, labels)
        dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
        ref = R.Loss(X, W, labels=labels)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    rX, bX, rW, bW = ref.grads(w, False)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N", [3, 140])
def test_widest_rows(E, dtype, N):
    K, V = 1 << 21, 40
    X, W, g = _head(N, K, V, dtype, seed=15)
    labels, w = _labels(N, V, g), _weight(N, g)
    loss, lse = E.espace_linear_cross_entropy(X, W, labels)
    dX, dW = E.espace_linear_cross_entropy_backward(w, X, W, labels, lse)
    ref = R.Loss(X, W, labels=labels)
    R.within(lse[:, None], ref.lse, ref.dlse, "lse")
    R.within(loss, ref.loss, ref.dloss, "loss")
    # beside the bound for roundings that all err one way, that of a random walk: sqrt(K)
    # half steps of sums up to 8 are 7e-4
    assert float((lse.double() - ref.lse[:, 0]).abs().max()) <= 1e-3
    rX, bX, rW, bW = ref.grads(w, N <= 128)
    R.within(dX, rX, bX, "dX")
    R.within(dW, rW, bW, "dW")
