"""Embedding lookup and its gradient by sorted tokens, against float64."""
import pytest
import torch

from tests import train_ref as R
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DT = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def E():
    need_gpu()
    import paper_2410_05437_amd as e
    return e


def _tokens(N, V, how, g):
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    if how == "same":
        t[:] = V - 1
    elif how == "frequent":
        t = (torch.rand(N, generator=g, device="cuda") ** 6 * V).long()
    elif how == "sorted":
        t = t.sort().values
    elif how == "padded":
        t[torch.rand(N, generator=g, device="cuda") < 0.5] = -1
        t[-1] = -(1 << 40)
    elif how == "outside":
        t[::3], t[1::3] = V, 1 << 40
    return t


@DT
@pytest.mark.parametrize("size", [(1, 1, 1), (1, 4096, 50), (16, 1003, 700), (333, 64, 5), (4097, 260, 3000)],
                         ids=lambda s: "N%d_K%d_V%d" % s)
@pytest.mark.parametrize("scale", [1.0, 45.25, -0.3])
def test_lookup(E, size, dtype, scale):
    N, K, V = size
    g = torch.Generator(device="cuda").manual_seed(N + K)
    table = R.padded(torch.randn(V, K, generator=g, device="cuda").to(dtype), dtype, extra=8)
    tokens = _tokens(N, V, "padded", g) if N > 2 else torch.zeros(N, dtype=torch.int64, device="cuda")
    X = R.out(N, K, dtype, "cuda", extra=16)
    E.espace_embedding(tokens, table, scale, X=X)
    ref = torch.where((tokens >= 0)[:, None], table[tokens.clamp(min=0)].float() * scale, 0.0).to(dtype)
    assert torch.equal(X, ref) and R.padding_untouched(X)
    if N > 2:
        tokens[2] = V
        X = E.espace_embedding(tokens, table, scale)
        assert bool(X[2].isnan().all()) and torch.equal(X[3:], ref[3:])


GRAD = [(1, 1, 1), (1, 4096, 50), (63, 1003, 700), (64, 8, 3), (1000, 64, 5), (2049, 2056, 300), (4097, 260, 3000),
        (3000, 24, 300001), (40000, 40, 1100), (8193, 40, 500), (20000, 132, 4096), (24576, 24, 1027)]


@DT
@pytest.mark.parametrize("how", ["random", "same", "frequent", "sorted", "padded", "outside"])
@pytest.mark.parametrize("size", GRAD, ids=lambda s: "N%d_K%d_V%d" % s)
def test_gradient(E, size, how, dtype):
    N, K, V = size
    g = torch.Generator(device="cuda").manual_seed(N + K + V)
    tokens = _tokens(N, V, how, g)
    dX = R.padded(torch.randn(N, K, generator=g, device="cuda").to(dtype), dtype, extra=8)
    scale = 2.7
    ws = torch.full((E.espace_embedding_workspace_bytes(N, K, V),), 255, dtype=torch.uint8, device="cuda")
    dE = R.out(V, K, dtype, "cuda", extra=8)
    E.espace_embedding_backward(tokens, dX, V, scale, dE=dE, workspace=ws)
    ref, bound = R.embedding_grad(tokens, dX, V, scale)
    R.within(dE, ref, bound, "dE")
    assert R.padding_untouched(dE)
    used = torch.zeros(V, dtype=torch.bool, device="cuda")
    used[tokens[(tokens >= 0) & (tokens < V)]] = True
    assert not dE[~used].any()
    again = E.espace_embedding_backward(tokens, dX, V, scale)
    assert torch.equal(dE, again)
    # onto a gradient that is there: rows that no token names keep their bits
    start = R.padded(torch.randn(V, K, generator=g, device="cuda").to(dtype), dtype)
    if V > 2:
        start[~used] = float("nan")
    both = R.padded(start, dtype)
    E.espace_embedding_backward(tokens, dX, V, scale, dE=both, accumulate=True)
    ref, bound = R.embedding_grad(tokens, dX, V, scale, start=start)
    R.within(both[used], ref[used], bound[used], "dE, accumulated")
    assert torch.equal(both[~used].view(torch.int16 if dtype == BF16 else torch.int32),
                       start[~used].view(torch.int16 if dtype == BF16 else torch.int32))
    assert R.padding_untouched(both)


def test_no_tokens(E):
    dE = R.out(5, 20, BF16, "cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    x = torch.empty((0, 20), dtype=BF16, device="cuda")
    E.espace_embedding_backward(none, x, 5, dE=dE)
    assert not dE.any() and R.padding_untouched(dE)
    dE.fill_(3.0)
    E.espace_embedding_backward(none, x, 5, dE=dE, accumulate=True)
    assert bool((dE == 3.0).all())
    assert E.espace_embedding(none, dE).shape == (0, 20)


def test_rows_past_2_gib(E):
    """A table whose rows lie past 2^31 bytes and 2^31 elements."""
    V, K = 70000, 32768
    table = torch.zeros((V, K), dtype=BF16, device="cuda")
    tokens = torch.tensor([V - 1, 3, 65537, V - 1], device="cuda")
    table[tokens] = torch.arange(1, 4, device="cuda").bfloat16()[[0, 1, 2, 0]][:, None]
    X = E.espace_embedding(tokens, table, 2.0)
    assert torch.equal(X, (2 * table[tokens].float()).bfloat16())
    E.espace_embedding_backward(tokens, X, V, 0.5, dE=table)
    assert [float(table[v].float().mean()) for v in (V - 1, 3, 65537, 4)] == [2.0, 2.0, 3.0, 0.0]
    assert float(table.abs().amax(1).float().sum()) == 7.0


@DT
def test_captured(E, dtype):
    N, K, V = 700, 264, 1500
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens = _tokens(N, V, "frequent", g)
    x = R.padded(torch.randn(N, K, generator=g, device="cuda").to(dtype), dtype)
    ws = torch.empty(E.espace_embedding_workspace_bytes(N, K, V), dtype=torch.uint8, device="cuda")

    def run(tokens):
        dE = E.espace_embedding_backward(tokens, x, V, 1.5, workspace=ws)
        return dE, E.espace_embedding(tokens, dE, 0.5)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run(tokens)
    torch.cuda.current_stream().wait_stream(stream)
    kept = tokens.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run(kept)
    for k in range(4):
        kept.copy_((tokens * (k + 1) + k) % V)
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        want = run((tokens * (k + 1) + k) % V)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


@DT
@pytest.mark.parametrize("N", [5, 64, 65, 300])
def test_gradient_of_the_largest_tables(E, dtype, N):
    """More entries than a launch has threads for; few tokens and more."""
    V, K = (1 << 29) + 7, 3
    g = torch.Generator(device="cuda").manual_seed(N)
    tokens = torch.randint(0, V, (N,), generator=g, device="cuda")
    tokens[0], tokens[1], tokens[2], tokens[3] = V - 1, 0, V - 1, -1
    dX = R.padded(torch.randn(N, K, generator=g, device="cuda").to(dtype), dtype)
    dE = R.out(V, K, dtype, "cuda")
    dE[:] = 1.0
    E.espace_embedding_backward(tokens, dX, V, dE=dE)
    named = tokens[tokens >= 0].unique()
    at = torch.searchsorted(named, tokens.clamp(min=0))
    ref, bound = R.embedding_grad(torch.where(tokens >= 0, at, -1), dX, named.numel(), 1.0)
    R.within(dE[named], ref, bound, "dE")
    dE[named] = 0.0
    assert not bool(dE.any())
    before = torch.randn(named.numel(), K, generator=g, device="cuda").to(dtype)
    dE[named] = before
    E.espace_embedding_backward(tokens, dX, V, dE=dE, accumulate=True)
    ref, bound = R.embedding_grad(torch.where(tokens >= 0, at, -1), dX, named.numel(), 1.0, start=before)
    R.within(dE[named], ref, bound, "dE")
    dE[named] = 0.0
    assert not bool(dE.any())


@DT
def test_most_tokens_a_call_takes(E, dtype):
    N, K, V = (1 << 21) - 1, 16, 5000
    g = torch.Generator(device="cuda").manual_seed(3)
    tokens = _tokens(N, V, "frequent", g)
    table = R.padded(torch.randn(V, K, generator=g, device="cuda").to(dtype), dtype)
    X = E.espace_embedding(tokens, table)
    assert torch.equal(X, table[tokens])
    dE = E.espace_embedding_backward(tokens, X, V)
    # (on the CPU: many float64 atomics on one row take minutes)
    ref, bound = R.embedding_grad(tokens.cpu(), X.cpu(), V, 1.0)
    R.within(dE.cpu(), ref, bound, "dE")


@DT
@pytest.mark.parametrize("N", [10, 100])
def test_widest_rows(E, dtype, N):
    K, V = 1 << 21, 23
    g = torch.Generator(device="cuda").manual_seed(N)
    tokens = _tokens(N, V, "frequent", g)
    table = torch.randn(V, K, generator=g, device="cuda").to(dtype)
    X = E.espace_embedding(tokens, table)
    assert torch.equal(X, table[tokens])
    dE = E.espace_embedding_backward(tokens, X, V)
    ref, bound = R.embedding_grad(tokens.cpu(), X.cpu(), V, 1.0)
    R.within(dE.cpu(), ref, bound, "dE")
