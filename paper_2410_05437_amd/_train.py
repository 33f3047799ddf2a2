"""ctypes binding of include/espace_train.h: the losses on the logits of a linear
head and the embedding, with their gradients (argument marshalling only, as
_lib.py)."""
import torch

from ._lib import (
    BF16,
    F32,
    EspaceError,
    _SIZE_MAX,
    _check,
    _dt,
    _mat,
    _on,
    _opt_out,
    _out,
    _same,
    _stream,
    _ws,
    lib,
)

MAX_TEACHER_ENTRIES = 1024


def espace_linear_loss_workspace_bytes(backward, N, K, V, T, dtype):
    """Workspace bytes of a loss (backward: of its gradients); T = 0: cross entropy."""
    n = lib.espace_linear_loss_workspace_bytes(1 if backward else 0, N, K, V, T, BF16 if dtype == torch.bfloat16 else F32)
    if n == _SIZE_MAX:
        raise EspaceError(2, "invalid sizes for workspace query")
    return n


def espace_embedding_workspace_bytes(N, K, V):
    """Workspace bytes of espace_embedding_backward."""
    n = lib.espace_embedding_workspace_bytes(N, K, V)
    if n == _SIZE_MAX:
        raise EspaceError(2, "invalid sizes for workspace query")
    return n


def _vec(t, name, dtype, size, device):
    """Pointer of a contiguous 1-D tensor of `size` elements."""
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, it must be {dtype}")
    if t.dim() != 1 or t.shape[0] != size or (size > 1 and t.stride(0) != 1):
        raise ValueError(f"{name} must be a contiguous 1-D tensor of {size} elements")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the operands on {device}")
    return t.data_ptr()


def _vec_out(t, name, size, device):
    if t is None:
        t = torch.empty(size, dtype=torch.float32, device=device)
    return t, _vec(t, name, torch.float32, size, device)


def _rows(t, name, dtype, shape, device):
    """(pointer, leading dimension) of a 2-D tensor with unit column stride."""
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, it must be {dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {shape[0]}x{shape[1]}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, the operands on {device}")
    if shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit column stride")
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else shape[1]


def _head(X, W):
    """(N, K, V) of activations X [N][K] and a head W [V][K]."""
    if X.dim() != 2 or W.dim() != 2 or X.shape[1] != W.shape[1]:
        raise ValueError(f"X {tuple(X.shape)} and W {tuple(W.shape)} must be [N][K] and [V][K]")
    _same(X, "X", (W, "W"))
    return X.shape[0], X.shape[1], W.shape[0]


def _loss_ws(workspace, backward, N, K, V, T, X):
    return _ws(workspace, espace_linear_loss_workspace_bytes(backward, N, K, V, T, X.dtype), X.device)


def espace_linear_cross_entropy(X, W, labels, loss=None, lse=None, workspace=None):
    """Cross entropy of the logits X·Wᵀ (X [N][K], W [V][K]) and the labels [N]
    (int64; below 0: no label, the token's loss is 0), without keeping the logits.
    Returns (loss [N], lse [N]), float32; lse is the log-sum-exp of each token's
    logits, which the backward pass takes."""
    N, K, V = _head(X, W)
    pl = _vec(labels, "labels", torch.int64, N, X.device)
    loss, po = _vec_out(loss, "loss", N, X.device)
    lse, pe = _vec_out(lse, "lse", N, X.device)
    ws, wsb = _loss_ws(workspace, False, N, K, V, 0, X)
    px, ldx = _mat(X, "X")
    pw, ldw = _mat(W, "W")
    with _on(X.device):
        _check(lib.espace_linear_cross_entropy(px, ldx, pw, ldw, pl, po, pe, N, K, V, _dt(X),
                                               ws.data_ptr() if ws is not None else 0, wsb, _stream(X.device)))
    return loss, lse


def espace_linear_cross_entropy_backward(dloss, X, W, labels, lse, dX=None, dW=None, want_dx=True, want_dw=True,
                                         workspace=None):
    """Gradients of Σ_n dloss[n]·loss[n] (dloss [N] float32: 1/N for a mean) with
    the forward pass's lse: dX [N][K] and dW [V][K].  Returns (dX, dW); either is
    None when not wanted."""
    N, K, V = _head(X, W)
    pd = _vec(dloss, "dloss", torch.float32, N, X.device)
    pl = _vec(labels, "labels", torch.int64, N, X.device)
    pe = _vec(lse, "lse", torch.float32, N, X.device)
    dX, pdx, lddx = _opt_out(dX, N, K, X, "dX", want_dx)
    dW, pdw, lddw = _opt_out(dW, V, K, X, "dW", want_dw)
    ws, wsb = _loss_ws(workspace, True, N, K, V, 0, X)
    px, ldx = _mat(X, "X")
    pw, ldw = _mat(W, "W")
    with _on(X.device):
        _check(lib.espace_linear_cross_entropy_backward(pd, px, ldx, pw, ldw, pl, pe, pdx, lddx, pdw, lddw, N, K, V,
                                                        _dt(X), ws.data_ptr() if ws is not None else 0, wsb,
                                                        _stream(X.device)))
    return dX, dW


def espace_linear_distillation(X, W, index, logits, temperature=1.0, loss=None, lse=None, picked=None,
                               workspace=None):
    """t²·KL(teacher ‖ student) at the temperature t, of a teacher known by its top
    logits: index [N][T] int64 (below 0: an empty place), logits [N][T] float32.
    The student's logits are X·Wᵀ / t (X [N][K], W [V][K]).  Returns (loss [N],
    lse [N], picked [N][T]), float32: lse of the student's logits and those at the
    teacher's entries, which the backward pass takes."""
    N, K, V = _head(X, W)
    T = index.shape[1] if index.dim() == 2 else 0
    pi, ldi = _rows(index, "index", torch.int64, (N, T), X.device)
    pz, ldl = _rows(logits, "logits", torch.float32, (N, T), X.device)
    loss, po = _vec_out(loss, "loss", N, X.device)
    lse, pe = _vec_out(lse, "lse", N, X.device)
    if picked is None:
        picked = torch.empty((N, T), dtype=torch.float32, device=X.device)
    pp, ldpk = _rows(picked, "picked", torch.float32, (N, T), X.device)
    ws, wsb = _loss_ws(workspace, False, N, K, V, T, X)
    px, ldx = _mat(X, "X")
    pw, ldw = _mat(W, "W")
    with _on(X.device):
        _check(lib.espace_linear_distillation(px, ldx, pw, ldw, pi, ldi, pz, ldl, po, pe, pp, ldpk, N, K, V, T,
                                              float(temperature), _dt(X), ws.data_ptr() if ws is not None else 0, wsb,
                                              _stream(X.device)))
    return loss, lse, picked


def espace_linear_distillation_backward(dloss, X, W, index, logits, lse, picked, temperature=1.0, dX=None, dW=None,
                                        want_dx=True, want_dw=True, workspace=None):
    """Gradients of Σ_n dloss[n]·loss[n] with the forward pass's lse and picked: dX
    [N][K] and dW [V][K].  Returns (dX, dW); either is None when not wanted."""
    N, K, V = _head(X, W)
    T = index.shape[1] if index.dim() == 2 else 0
    pd = _vec(dloss, "dloss", torch.float32, N, X.device)
    pi, ldi = _rows(index, "index", torch.int64, (N, T), X.device)
    pz, ldl = _rows(logits, "logits", torch.float32, (N, T), X.device)
    pe = _vec(lse, "lse", torch.float32, N, X.device)
    pp, ldpk = _rows(picked, "picked", torch.float32, (N, T), X.device)
    dX, pdx, lddx = _opt_out(dX, N, K, X, "dX", want_dx)
    dW, pdw, lddw = _opt_out(dW, V, K, X, "dW", want_dw)
    ws, wsb = _loss_ws(workspace, True, N, K, V, T, X)
    px, ldx = _mat(X, "X")
    pw, ldw = _mat(W, "W")
    with _on(X.device):
        _check(lib.espace_linear_distillation_backward(pd, px, ldx, pw, ldw, pi, ldi, pz, ldl, pe, pp, ldpk, pdx, lddx,
                                                       pdw, lddw, N, K, V, T, float(temperature), _dt(X),
                                                       ws.data_ptr() if ws is not None else 0, wsb,
                                                       _stream(X.device)))
    return dX, dW


def espace_embedding(tokens, E, scale=1.0, X=None):
    """X[n] = scale·E[tokens[n]]  (tokens [N] int64, E [V][K] -> X [N][K]); zeros
    for a token below 0, NaN for one past the table."""
    if tokens.dim() != 1 or E.dim() != 2:
        raise ValueError("tokens must be 1-D and E 2-D")
    N, (V, K) = tokens.shape[0], E.shape
    pt = _vec(tokens, "tokens", torch.int64, N, E.device)
    X = _out(X, N, K, E, "X")
    pe, lde = _mat(E, "E")
    px, ldx = _mat(X, "X")
    with _on(E.device):
        _check(lib.espace_embedding(pt, pe, lde, px, ldx, N, K, V, float(scale), _dt(E), _stream(E.device)))
    return X


def espace_embedding_backward(tokens, dX, V, scale=1.0, dE=None, accumulate=False, workspace=None):
    """dE[v] = scale·Σ dX[n] over the tokens n = v (tokens [N] int64, dX [N][K] -> dE
    [V][K]); with `accumulate` added to dE, whose other rows stay as they are."""
    if tokens.dim() != 1 or dX.dim() != 2:
        raise ValueError("tokens must be 1-D and dX 2-D")
    if accumulate and dE is None:
        raise ValueError("accumulate needs dE")
    N, K = dX.shape
    pt = _vec(tokens, "tokens", torch.int64, N, dX.device)
    dE = _out(dE, V, K, dX, "dE")
    ws, wsb = _ws(workspace, espace_embedding_workspace_bytes(N, K, V), dX.device)
    px, lddx = _mat(dX, "dX")
    pe, ldde = _mat(dE, "dE")
    with _on(dX.device):
        _check(lib.espace_embedding_backward(pt, px, lddx, pe, ldde, N, K, V, float(scale), 1 if accumulate else 0,
                                             _dt(dX), ws.data_ptr() if ws is not None else 0, wsb,
                                             _stream(dX.device)))
    return dE
