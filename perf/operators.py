"""The two ends of a model in retraining, as cases for timing: token embeddings
at its input; at its output the head's product with the loss on its logits, by
labels (cross entropy) or by a teacher's top logits (distillation).  A layer
that was projected is retrained between them, and the gradients that the loss
sends back are what the NL-MSE calibration reads.

Letters as elsewhere: K features, N tokens, V entries of the vocabulary, T
teacher entries a token.  Kinds:

  score    loss and log-sum-exp of every token by its label (evaluation)
  step     the same, then dX and dW of the weighted sum of the losses
  distill  loss, log-sum-exp and the student's logits at the entries by the
           teacher's top logits, then dX and dW
  distill_score   the same without the gradients
  lookup   embedding rows of the tokens, scaled
  embgrad  gradient of the embedding from that of its outputs

Formulas, with s_v = x·w_v:

  score    lse = log Σ_v exp(s_v);  loss = lse - s_label  (0 without a label)
  distill  q = softmax(s / t), p = softmax over the teacher's entries of its
           logits / t;  loss = t² Σ_j p_j (log p_j - log q_{i_j});  lse that of
           s / t, picked_j = s_{i_j} / t (0 where there is no entry); a token
           without an entry has loss 0
  step     G = weight·(q - onehot(label)), or weight·t·(q - Σ_j p_j onehot(i_j));
           dX = G·W, dW = Gᵀ·X
  lookup   X[n] = scale·E[token_n]  (zeros for a padding token, one below 0)
  embgrad  dE[v] = scale·Σ_{n: token_n = v} dX[n]
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64


def listed():
    return [
        # evaluation of a tiny fp32 model (the repository's tiny width): the calls' latency
        dict(name="score_f32_small", kind="score", dtype="f32", N=100, K=256, V=1000, T=0, t=1.0),
        # one decoded token scored against a Llama2-7B width head
        dict(name="score_n1", kind="score", dtype="bf16", N=1, K=4096, V=32000, T=0, t=1.0),
        # perplexity of a short prompt, GPT3-22B width, odd vocabulary
        dict(name="score_n333", kind="score", dtype="bf16", N=333, K=6144, V=50257, T=0, t=1.0),
        # a training step's head in fp32, ragged sizes
        dict(name="step_f32", kind="step", dtype="f32", N=601, K=1000, V=5003, T=0, t=1.0),
        # a retraining step's head: Llama2-7B width, one sequence
        dict(name="step_n4096", kind="step", dtype="bf16", N=4096, K=4096, V=32000, T=0, t=1.0),
        # the largest: GPT3-22B width, odd vocabulary, its benchmark's 8192 tokens
        dict(name="step_n8192", kind="step", dtype="bf16", N=8192, K=6144, V=50257, T=0, t=1.0),
        # distillation of a small model, one short text
        dict(name="distill_small", kind="distill", dtype="bf16", N=65, K=256, V=1000, T=8, t=1.0),
        # distillation through a head that was itself projected (K = its kept components)
        dict(name="distill_n4096", kind="distill", dtype="bf16", N=4096, K=1536, V=32000, T=64, t=2.0),
        # inputs of one decoded token for each of 16 sequences
        dict(name="lookup_n16", kind="lookup", dtype="bf16", N=16, K=4096, V=32000, T=0, t=1.0),
        # inputs of a prefill, GPT3-22B width
        dict(name="lookup_n8192", kind="lookup", dtype="bf16", N=8192, K=6144, V=50257, T=0, t=78.4),
        # gradient of a step's embedding, Llama2-7B width
        dict(name="embgrad_n4096", kind="embgrad", dtype="bf16", N=4096, K=4096, V=32000, T=0, t=1.0),
        # the same for many short fp32 rows: more tokens than the vocabulary has
        dict(name="embgrad_f32", kind="embgrad", dtype="f32", N=20011, K=500, V=5003, T=0, t=22.4),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _size(rng, lo, hi):
    """A size between lo and hi: a multiple of 128, of 8, or any number."""
    v = _log(rng, lo, hi)
    step = rng.choice([128, 8, 1])
    return min(hi, max(lo, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["score"] * 3 + ["step"] * 4 + ["distill"] * 3 + ["distill_score", "lookup", "lookup", "embgrad", "embgrad"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind in ("lookup", "embgrad"):
        return dict(kind=kind, dtype=dtype, N=int(_log(rng, 1, 32768)), K=_size(rng, 64, 8192),
                    V=_size(rng, 500, 65536), T=0, t=rng.choice([1.0, 22.4]))
    T = int(_log(rng, 1, 128)) if kind.startswith("distill") else 0
    t = rng.choice([1.0, 2.0, 4.0]) if T else 1.0
    while True:
        big = dtype == "bf16"
        N = int(_log(rng, 1 if kind == "score" else 16, 8192 if big else 2048))
        K, V = _size(rng, 64, 8192 if big else 2048), _size(rng, 500, 131072 if big else 16384)
        if N * K * V <= (2.5e12 if big else 1e10) and N * V <= 1 << 29:
            return dict(kind=kind, dtype=dtype, N=N, K=K, V=V, T=T, t=t)


# ---- inputs --------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 1000003 + 29)


def _normal(g, rows, cols):
    return torch.randn((rows, cols), generator=g, device=DEV, dtype=F32)


def _mat(t, dtype):
    """The matrix with its rows padded to 16 bytes, as this library's callers keep
    matrices."""
    rows, cols = t.shape
    a = 8 if dtype == BF16 else 4
    out = torch.zeros((rows, (cols + a - 1) // a * a), dtype=dtype, device=DEV)[:, :cols]
    return out.copy_(t)


def _tokens(g, N, V):
    """Token numbers as texts have them: the v-th about as often as 1 / v."""
    u = torch.rand(N, generator=g, device=DEV, dtype=F64)
    return (torch.exp(u * math.log(V + 1)).floor().long() - 1).clamp_(0, V - 1)


def _inputs(case, seed):
    g = _gen(seed)
    kind, N, K, V, T = (case[k] for k in ("kind", "N", "K", "V", "T"))
    dt = F32 if case["dtype"] == "f32" else BF16
    if kind in ("lookup", "embgrad"):
        tokens = _tokens(g, N, V)
        if N > 8:    # a batch's padding
            tokens[torch.rand(N, generator=g, device=DEV) < 0.03] = -1
        if kind == "lookup":
            return dict(tokens=tokens, E=_mat(_normal(g, V, K) * K ** -0.5, dt))
        return dict(tokens=tokens, dX=_mat(_normal(g, N, K) * 1e-3, dt))
    # outputs of the last norm layer: channels of unequal size; logits of standard deviation 2
    s = torch.exp(0.5 * _normal(g, 1, K))
    x = _normal(g, N, K) * s
    X = _mat(x * (K ** 0.5 / x.norm(dim=1, keepdim=True)), dt)
    W = _mat(_normal(g, V, K) * (2.0 * K ** -0.5), dt)
    out = dict(X=X, W=W)
    # tokens of the prompt have no loss: a tenth of them
    masked = torch.rand(N, generator=g, device=DEV) < (0.1 if N > 8 else 0.0)
    if T:
        # the teacher: the student's logits, disturbed; its T largest.  Some tokens
        # keep fewer (a cut by probability), the rest of their places are -1
        a, b = X.bfloat16(), W.bfloat16()
        z = torch.mm(a, b.t()).float()
        z += torch.randn(z.shape, generator=g, device=DEV, dtype=F32)
        logits, index = z.topk(min(T, V), dim=1)
        del z
        fewer = torch.rand(N, generator=g, device=DEV) < 0.2
        keep = 1 + torch.randint(0, index.shape[1], (N,), generator=g, device=DEV)
        keep = torch.where(fewer, keep, index.shape[1])
        keep = torch.where(masked, 0, keep)
        index[torch.arange(index.shape[1], device=DEV)[None, :] >= keep[:, None]] = -1
        out |= dict(index=index.contiguous(), logits=logits.contiguous())
    else:
        labels = _tokens(g, N, V)
        labels[masked] = -100
        out["labels"] = labels
    # the mean over the tokens that have a loss
    counted = (~masked).to(F32)
    out["weight"] = counted / counted.sum().clamp(min=1.0)
    return out


def prepare(case, seed):
    """Activations, weights and labels as a training program holds them."""
    return dict(case=case, **_inputs(case, seed))


# ---- one pass --------------------------------------------------------------------


def _own(s):
    import paper_2410_05437_amd as espace

    kind, t = s["case"]["kind"], s["case"]["t"]
    if kind == "lookup":
        return espace.espace_embedding(s["tokens"], s["E"], scale=t)
    if kind == "embgrad":
        return espace.espace_embedding_backward(s["tokens"], s["dX"], s["case"]["V"], scale=t)
    X, W = s["X"], s["W"]
    if kind in ("score", "step"):
        loss, lse = espace.espace_linear_cross_entropy(X, W, s["labels"])
        if kind == "score":
            return dict(loss=loss, lse=lse)
        dX, dW = espace.espace_linear_cross_entropy_backward(s["weight"], X, W, s["labels"], lse)
    else:
        loss, lse, picked = espace.espace_linear_distillation(X, W, s["index"], s["logits"], temperature=t)
        if kind == "distill_score":
            return dict(loss=loss, lse=lse, picked=picked)
        dX, dW = espace.espace_linear_distillation_backward(s["weight"], X, W, s["index"], s["logits"], lse, picked,
                                                            temperature=t)
        return dict(loss=loss, lse=lse, picked=picked, dX=dX, dW=dW)
    return dict(loss=loss, lse=lse, dX=dX, dW=dW)


def _teacher(index, logits, t):
    """(entries' probabilities, their logarithms, places with an entry) of each token."""
    there = index >= 0
    z = torch.where(there, logits / t, -math.inf)
    z = z - z.amax(1, keepdim=True).clamp(min=torch.finfo(z.dtype).min)
    e = torch.where(there, torch.exp(z), 0.0)
    total = e.sum(1, keepdim=True)
    p = e / total.clamp(min=torch.finfo(z.dtype).tiny)
    return p, torch.where(there, z - torch.log(total), 0.0), there


def run(s):
    if own:
        return _own(s)
    case = s["case"]
    kind, t = case["kind"], case["t"]
    if kind == "lookup":
        tokens = s["tokens"]
        rows = s["E"][tokens.clamp(min=0)].float() * t
        return torch.where((tokens >= 0)[:, None], rows, 0.0).to(s["E"].dtype)
    if kind == "embgrad":
        there = s["tokens"] >= 0
        dE = torch.zeros((case["V"], case["K"]), dtype=F32, device=DEV)
        dE.index_add_(0, s["tokens"].clamp(min=0), torch.where(there[:, None], s["dX"].float(), 0.0))
        return (dE * t).to(s["dX"].dtype)
    X, W = s["X"].float(), s["W"].float()
    S = torch.mm(X, W.t())
    if t != 1.0:
        S = S / t
    top = S.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(S - top).sum(1, keepdim=True))
    if kind in ("score", "step"):
        there = (s["labels"] >= 0)[:, None]
        at, p = s["labels"].clamp(min=0)[:, None], there.to(F32)
        loss = torch.where(there, lse - S.gather(1, at), 0.0)
    else:
        p, logp, there = _teacher(s["index"], s["logits"], t)
        at = s["index"].clamp(min=0)
        loss = t * t * (p * torch.where(there, logp - S.gather(1, at) + lse, 0.0)).sum(1, keepdim=True)
    out = dict(loss=loss[:, 0], lse=lse[:, 0])
    if kind.startswith("distill"):
        out["picked"] = torch.where(there, S.gather(1, at), 0.0)
    if not kind.endswith("score"):
        G = torch.exp(S - lse)
        G = torch.where(there.any(1, keepdim=True), G, 0.0)
        G = G.scatter_add(1, at, -p) * (t * s["weight"][:, None])
        out |= dict(dX=torch.mm(G, W).to(s["X"].dtype), dW=torch.mm(G.t(), X).to(s["X"].dtype))
    return out


# ---- what a pass cannot do without, and its exact result ---------------------------


def work(case):
    kind, N, K, V, T = (case[k] for k in ("kind", "N", "K", "V", "T"))
    e = 4 if case["dtype"] == "f32" else 2
    if kind == "lookup":
        return dict(flops=N * K, bytes=2 * e * N * K + 8 * N)
    if kind == "embgrad":
        return dict(flops=N * K, bytes=e * (N * K + V * K) + 8 * N)
    read = e * (N * K + V * K) + N * (16 * T if T else 8) + 8 * N
    if kind.endswith("score"):
        return dict(flops=2 * N * V * K, bytes=read)
    # the logits' product and the two gradients'
    return dict(flops=6 * N * V * K, bytes=read + e * (N * K + V * K) + 4 * N)


def exact(case, seed):
    s = {k: v.to(F64) if v.is_floating_point() else v for k, v in _inputs(case, seed).items()}
    kind, t, N, K, V = (case[k] for k in ("kind", "t", "N", "K", "V"))
    if kind == "lookup":
        rows = torch.cat([s["E"], torch.zeros((1, K), dtype=F64, device=DEV)])
        return torch.index_select(rows, 0, torch.where(s["tokens"] < 0, V, s["tokens"])) * t
    if kind == "embgrad":
        # tokens in order, differences of running sums at the ends of each run
        order = s["tokens"].argsort(stable=True)
        ends = torch.searchsorted(s["tokens"][order].contiguous(), torch.arange(-1, V, device=DEV), right=True)
        sums = torch.cat([torch.zeros((1, K), dtype=F64, device=DEV), s["dX"][order].cumsum(0)])[ends]
        return (sums[1:] - sums[:-1]) * t
    grads = not kind.endswith("score")
    loss, lse, picked = [], [], []
    dX, dW = [], torch.zeros((V, K), dtype=F64, device=DEV)
    for n0 in range(0, N, 2048):
        rows = slice(n0, n0 + 2048)
        x = s["X"][rows]
        logq = torch.log_softmax(torch.mm(x, s["W"].t()) / t, dim=1)
        lse.append(torch.logsumexp(torch.mm(x, s["W"].t()) / t, dim=1))
        target = torch.zeros_like(logq)
        if "labels" in s:
            hit = torch.nonzero(s["labels"][rows] >= 0)[:, 0]
            target[hit, s["labels"][rows][hit]] = 1.0
        else:
            n, j = torch.nonzero(s["index"][rows] >= 0, as_tuple=True)
            z = torch.full(s["index"][rows].shape, -math.inf, dtype=F64, device=DEV)
            z[n, j] = s["logits"][rows][n, j] / t
            target[n, s["index"][rows][n, j]] = torch.softmax(z, dim=1)[n, j]
            at = torch.zeros_like(z)
            at[n, j] = (torch.mm(x, s["W"].t()) / t)[n, s["index"][rows][n, j]]
            picked.append(at)
        loss.append(t * t * (torch.xlogy(target, target) - target * logq).sum(1))
        if grads:
            G = (torch.exp(logq) * target.sum(1, keepdim=True) - target) * (t * s["weight"][rows][:, None])
            dX.append(torch.mm(G, s["W"]))
            dW += torch.mm(G.t(), x)
        del logq, target
    out = dict(loss=torch.cat(loss), lse=torch.cat(lse))
    if picked:
        out["picked"] = torch.cat(picked)
    if grads:
        out |= dict(dX=torch.cat(dX), dW=dW)
    return out
