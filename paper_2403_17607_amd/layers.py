"""Layer norm, dense layers of any width, and losses over a vocabulary.

Like FusedMLP, each class holds a shape and no device memory; weights,
workspaces and outputs are the caller's tensors (outputs that are not given
are allocated).  Matrices are bf16 (or fp32 where stated), one row per sample
or token, and may be slices of wider ones: elements of a row are consecutive,
rows any distance apart.  A workspace belongs to one call at a time; calls on
other streams need their own.  Results are bitwise the same from run to run.

Example::

    norm, up = LayerNorm(1024), Dense(1024, 4096, "gelu")
    H = norm.forward(X, gamma, beta, stats=stats)
    Y = up.forward(W, H, bias, stash=stash, ws=ws)
    dH, dW, db = up.backward(W, H, dY, ws, stash=stash)
    dX, dgamma, dbeta = norm.backward(X, gamma, stats, dH, ws_norm)

    head = SoftmaxHead(dim=128, vocab=50000)
    dH, dW, loss = head.cross_entropy_step(W, H, target, head.workspace(M))
"""
from __future__ import annotations

import torch

import paper_2403_17607_amd as _base

MLP_BF16 = 0
MLP_FP32 = 1
MLP_MAX_DIM = 1 << 22

ACTIVATIONS_DENSE = {"linear": 0, "relu": 1, "sigmoid": 2, "sine": 3, "gelu": 4, "silu": 5}

_TYPES = {torch.bfloat16: MLP_BF16, torch.float32: MLP_FP32}


def _matrix(t, name, rows, cols, dtypes=(torch.bfloat16,), device=None) -> int:
    """Check a [rows, cols] GPU matrix whose rows are consecutive elements;
    returns its row stride.  As with the other checks of this package, these
    stand between a mistyped or short tensor and an access out of bounds."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be one of {[str(d) for d in dtypes]}, got {t.dtype}")
    if t.shape != (rows, cols):
        raise ValueError(f"{name} must have shape {(rows, cols)}, got {tuple(t.shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the other arguments on {device}")
    if rows == 0:
        return cols
    ld, unit = t.stride()
    if cols > 1 and unit != 1:
        raise ValueError(f"the elements of a row of {name} must be consecutive")
    if rows == 1:
        return cols
    if ld < cols:
        raise ValueError(f"the rows of {name} overlap (row stride {ld}, {cols} columns)")
    return ld


def _vector(t, name, n, device, dtype=torch.float32):
    if t is None:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == (n,) and t.device == device and t.is_contiguous()):
        _base._require(t, name, dtype, shape=(n,), device=device)  # says what is wrong
    return t.data_ptr()


def _out(t, name, rows, cols, dtype, device):
    """The output matrix `name`, allocated unless given, and its row stride."""
    if t is None:
        if dtype not in _TYPES:
            raise ValueError(f"{name} must be bfloat16 or float32, got {dtype}")
        return torch.empty(rows, cols, dtype=dtype, device=device), cols
    return t, _matrix(t, name, rows, cols, _TYPES, device)


def _rows(X, name, cols) -> int:
    if not isinstance(X, torch.Tensor) or X.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor [M, {cols}]")
    return X.shape[0]


def _dim(n, name) -> int:
    if not isinstance(n, int) or isinstance(n, bool) or not 1 <= n <= MLP_MAX_DIM:
        raise ValueError(f"{name} must be an int in [1, {MLP_MAX_DIM}], got {n!r}")
    return n


# the current device's index; torch.cuda.current_device() makes sure of the
# initialisation first, which a tensor on the GPU has done
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _run(fn, dev, *args) -> None:
    """Call fn(*args, stream) with `dev` as the current device."""
    if dev.index == _current_device():
        rc = fn(*args, _base._stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _base._stream(dev))
    if rc != 0:
        _base._check(rc)


class _Layer:
    # the last workspace size asked for, with its arguments; that of forward calls
    # apart, so that a training step's two sides do not replace each other's
    _need = (None, 0)
    _need_infer = (None, 0)

    def _ws_bytes(self, *key) -> int:
        infer = key[1:2] == (_base.MLP_MODE_INFER,)
        need = self._need_infer if infer else self._need  # read once: other threads may set it
        if need[0] != key:
            need = (key, self.workspace_bytes(*key))
            if infer:
                self._need_infer = need
            else:
                self._need = need
        return need[1]

    def workspace_bytes(self, M: int, mode: int = _base.MLP_MODE_TRAIN) -> int:
        raise NotImplementedError

    def workspace(self, M: int, device="cuda", mode: int = _base.MLP_MODE_TRAIN) -> torch.Tensor:
        """A workspace for a batch of exactly M rows."""
        return torch.empty(max(self.workspace_bytes(M, mode), 1), dtype=torch.uint8, device=device)

    def _ws(self, ws, need, device):
        if need == 0 and ws is None:
            return None
        _base._require(ws, "ws", torch.uint8, min_numel=need, device=device)
        return ws.data_ptr()


class LayerNorm(_Layer):
    """Layer norm of rows of `dim` elements: Y = (X - mean) / sqrt(var + eps) * gamma + beta."""

    def __init__(self, dim: int, eps: float = 1e-5):
        self.dim = _dim(dim, "dim")
        if not 0.0 < eps < float("inf"):
            raise ValueError("eps must be positive and finite")
        self.eps = float(eps)

    def workspace_bytes(self, M: int, mode: int = _base.MLP_MODE_TRAIN) -> int:
        return int(_base.lib().mlp_layer_norm_workspace_bytes(M, self.dim, mode))

    def forward(self, X, gamma=None, beta=None, Y=None, stats=None, dtype=None) -> torch.Tensor:
        """X [M, dim] (bf16 or fp32) -> Y of `dtype` (default: X's).  gamma and
        beta: fp32 [dim], or None for ones and zeros.  stats: fp32 [M, 2],
        receives the mean and 1 / std of every row for backward()."""
        M, n = _rows(X, "X", self.dim), self.dim
        ldx, dev = _matrix(X, "X", M, n, _TYPES), X.device
        Y, ldy = _out(Y, "Y", M, n, dtype or X.dtype, dev)
        if stats is not None:
            _base._require(stats, "stats", torch.float32, shape=(M, 2), device=dev)
        _run(
            _base.lib().mlp_layer_norm_forward, dev, X.data_ptr(), _TYPES[X.dtype], ldx, _vector(gamma, "gamma", n, dev), _vector(beta, "beta", n, dev),
            Y.data_ptr(), _TYPES[Y.dtype], ldy, None if stats is None else stats.data_ptr(), M, n, self.eps)
        return Y

    def backward(self, X, gamma, stats, dY, ws, dX=None, dgamma=None, dbeta=None, dtype=None):
        """The gradients from dY [M, dim] and the forward's X and stats:
        (dX of `dtype` (default: X's), dgamma, dbeta (fp32 [dim]))."""
        M, n = _rows(X, "X", self.dim), self.dim
        ldx, dev = _matrix(X, "X", M, n, _TYPES), X.device
        lddy = _matrix(dY, "dY", M, n, _TYPES, dev)
        _base._require(stats, "stats", torch.float32, shape=(M, 2), device=dev)
        dX, lddx = _out(dX, "dX", M, n, dtype or X.dtype, dev)
        dgamma = torch.empty(n, dtype=torch.float32, device=dev) if dgamma is None else dgamma
        dbeta = torch.empty(n, dtype=torch.float32, device=dev) if dbeta is None else dbeta
        _run(
            _base.lib().mlp_layer_norm_backward, dev, X.data_ptr(), _TYPES[X.dtype], ldx, _vector(gamma, "gamma", n, dev), stats.data_ptr(), dY.data_ptr(),
            _TYPES[dY.dtype], lddy, dX.data_ptr(), _TYPES[dX.dtype], lddx, _vector(dgamma, "dgamma", n, dev),
            _vector(dbeta, "dbeta", n, dev), M, n, self._ws(ws, self._ws_bytes(M), dev))
        return dX, dgamma, dbeta


class Dense(_Layer):
    """One layer of any width: Y = act(X W + bias) + residual, with W bf16
    [in_dim, out_dim] and `activation` one of linear, relu, sigmoid, sine,
    gelu (x Phi(x)) and silu."""

    def __init__(self, in_dim: int, out_dim: int, activation="linear"):
        self.in_dim, self.out_dim = _dim(in_dim, "in_dim"), _dim(out_dim, "out_dim")
        if isinstance(activation, str):
            if activation not in ACTIVATIONS_DENSE:
                raise ValueError(f"activation must be one of {sorted(ACTIVATIONS_DENSE)}, got {activation!r}")
            activation = ACTIVATIONS_DENSE[activation]
        if activation not in ACTIVATIONS_DENSE.values():
            raise ValueError(f"unknown activation {activation!r}")
        self.activation = activation

    def workspace_bytes(self, M: int, mode: int = _base.MLP_MODE_TRAIN) -> int:
        return int(_base.lib().mlp_dense_workspace_bytes(M, self.in_dim, self.out_dim, mode))

    def stash(self, M: int, device="cuda"):
        """What forward() keeps for backward(): fp32 [M, out_dim]; None for a
        linear layer, which keeps nothing."""
        if self.activation == 0:
            return None
        return torch.empty(M, self.out_dim, dtype=torch.float32, device=device)

    def forward(self, W, X, bias=None, residual=None, Y=None, stash=None, ws=None, dtype=None) -> torch.Tensor:
        """X bf16 [M, in_dim] -> Y [M, out_dim] of `dtype` (bf16 unless the
        residual says otherwise; the residual has Y's type and may be Y).
        bias: fp32 [out_dim].  ws: a workspace of either mode, needed where
        workspace_bytes(M, MLP_MODE_INFER) is not 0."""
        M, k, n = _rows(X, "X", self.in_dim), self.in_dim, self.out_dim
        ldx, dev = _matrix(X, "X", M, k), X.device
        ldw = _matrix(W, "W", k, n, device=dev)
        if dtype is None:
            dtype = residual.dtype if isinstance(residual, torch.Tensor) else torch.bfloat16
        Y, ldy = _out(Y, "Y", M, n, dtype, dev)
        ldr = 0 if residual is None else _matrix(residual, "residual", M, n, (Y.dtype,), dev)
        if stash is not None:
            _base._require(stash, "stash", torch.float32, shape=(M, n), device=dev)
        L = _base.lib()
        _run(
            L.mlp_dense_forward, dev, X.data_ptr(), ldx, W.data_ptr(), ldw, _vector(bias, "bias", n, dev), self.activation,
            None if residual is None else residual.data_ptr(), ldr, Y.data_ptr(), _TYPES[Y.dtype], ldy,
            None if stash is None else stash.data_ptr(), M, k, n,
            self._ws(ws, self._ws_bytes(M, _base.MLP_MODE_INFER), dev))
        return Y

    def backward(self, W, X, dY, ws, stash=None, dX=None, dW=None, db=None, dtype=torch.float32, input_gradient=True):
        """The gradients from dY [M, out_dim] (bf16 or fp32) and the forward's
        W, X and stash: (dX [M, in_dim], dW [in_dim, out_dim], both of
        `dtype`, db fp32 [out_dim]).  input_gradient=False: no dX (None).
        The residual's gradient is dY."""
        M, k, n = _rows(X, "X", self.in_dim), self.in_dim, self.out_dim
        ldx, dev = _matrix(X, "X", M, k), X.device
        ldw = _matrix(W, "W", k, n, device=dev)
        lddy = _matrix(dY, "dY", M, n, _TYPES, dev)
        if self.activation != 0:
            _base._require(stash, "stash", torch.float32, shape=(M, n), device=dev)
        lddx = k
        if input_gradient:
            dX, lddx = _out(dX, "dX", M, k, dtype, dev)
        elif dX is not None:
            raise ValueError("dX was given, but input_gradient is False")
        dW, lddw = _out(dW, "dW", k, n, dtype, dev)
        db = torch.empty(n, dtype=torch.float32, device=dev) if db is None else db
        L = _base.lib()
        _run(
            L.mlp_dense_backward, dev, X.data_ptr(), ldx, W.data_ptr(), ldw, self.activation, None if stash is None else stash.data_ptr(),
            dY.data_ptr(), _TYPES[dY.dtype], lddy, None if dX is None else dX.data_ptr(),
            0 if dX is None else _TYPES[dX.dtype], lddx, dW.data_ptr(), _TYPES[dW.dtype], lddw,
            _vector(db, "db", n, dev), M, k, n, self._ws(ws, self._ws_bytes(M), dev))
        return dX, dW, db


class SoftmaxHead(_Layer):
    """Losses of the logits H W, W bf16 [dim, vocab], over a vocabulary.  The
    logits are not stored: the loss alone keeps two sums per row and run of
    columns, the ..._step calls the probabilities of a piece of the vocabulary
    in 16 bits, up to 1 GiB (or 1024 columns) in the workspace.  These also
    return the gradients of the mean loss, as train_step does; dH is what a net
    that made H takes as its dY."""

    def __init__(self, dim: int, vocab: int):
        self.dim, self.vocab = _dim(dim, "dim"), _dim(vocab, "vocab")

    def workspace_bytes(self, M: int, mode: int = _base.MLP_MODE_TRAIN, top: int = 1) -> int:
        return int(_base.lib().mlp_head_workspace_bytes(M, self.dim, self.vocab, top, mode))

    def workspace(self, M: int, device="cuda", mode: int = _base.MLP_MODE_TRAIN, top: int = 1) -> torch.Tensor:
        """A workspace for a batch of exactly M rows (and teacher lists of `top`
        entries).  MLP_MODE_INFER suffices for calls without gradients."""
        return torch.empty(max(self.workspace_bytes(M, mode, top), 1), dtype=torch.uint8, device=device)

    def _call(self, fn, W, H, extra, top, ws, grads, loss, row_loss, dH, dW, dtype):
        M, d, v = _rows(H, "H", self.dim), self.dim, self.vocab
        ldh, dev = _matrix(H, "H", M, d), H.device
        ldw = _matrix(W, "W", d, v, device=dev)
        args = extra(M, dev)
        if loss is None:
            loss = torch.empty(1, dtype=torch.float32, device=dev)
        _base._require(loss, "loss", torch.float32, shape=(1,), device=dev)
        lddh, lddw, pH, pW, tH, tW = d, v, None, None, 0, 0
        if grads:
            dH, lddh = _out(dH, "dH", M, d, dtype, dev)
            dW, lddw = _out(dW, "dW", d, v, dtype, dev)
            pH, pW, tH, tW = dH.data_ptr(), dW.data_ptr(), _TYPES[dH.dtype], _TYPES[dW.dtype]
            if M == 0:
                pH = pW  # an empty tensor has no address; nothing is written to it
        mode = _base.MLP_MODE_TRAIN if grads else _base.MLP_MODE_INFER
        _run(
            fn, dev, H.data_ptr(), ldh, W.data_ptr(), ldw, *args, loss.data_ptr(),
            _vector(row_loss, "row_loss", M, dev), pH, tH, lddh, pW, tW, lddw, M, d, v,
            self._ws(ws, self._ws_bytes(M, mode, top), dev))
        return (dH, dW, loss) if grads else loss

    def _target(self, target, ignore_index):
        def extra(M, dev):
            return _vector(target, "target", M, dev, torch.int64), ignore_index
        if target is None:
            raise ValueError("target must be a torch.Tensor")
        return extra

    def _teacher(self, index, logits, temperature):
        if not isinstance(index, torch.Tensor) or index.dim() != 2:
            raise ValueError("index must be a 2-D tensor [M, top]")
        top = index.shape[1]

        def extra(M, dev):
            _base._require(index, "index", torch.int64, shape=(M, top), device=dev)
            if not isinstance(logits, torch.Tensor) or logits.dtype not in _TYPES:
                raise ValueError("logits must be a bfloat16 or float32 tensor")
            _base._require(logits, "logits", logits.dtype, shape=(M, top), device=dev)
            return index.data_ptr(), logits.data_ptr(), _TYPES[logits.dtype], top, temperature
        return extra, top

    def cross_entropy(self, W, H, target, ws, ignore_index: int = -100, loss=None, row_loss=None):
        """Mean over the rows with target != ignore_index of
        -log softmax(H W)[target] (0 if there is none), as a device tensor [1].
        H bf16 [M, dim]; target int64 [M], 0 .. vocab - 1 or ignore_index, any
        other value makes the loss NaN.  row_loss: fp32 [M], the loss of every row."""
        return self._call(_base.lib().mlp_cross_entropy, W, H, self._target(target, ignore_index), 1, ws, False, loss,
                          row_loss, None, None, None)

    def cross_entropy_step(self, W, H, target, ws, ignore_index: int = -100, loss=None, row_loss=None, dH=None,
                           dW=None, dtype=torch.float32):
        """cross_entropy() and its gradients: (dH [M, dim], dW [dim, vocab], loss)."""
        return self._call(_base.lib().mlp_cross_entropy, W, H, self._target(target, ignore_index), 1, ws, True, loss,
                          row_loss, dH, dW, dtype)

    def distill(self, W, H, index, logits, ws, temperature: float = 1.0, loss=None, row_loss=None):
        """Mean over the rows that have an entry of temperature^2
        KL(softmax(logits / temperature) || softmax(H W / temperature)), the
        teacher's distribution over a row's entries alone.  index int64 [M,
        top] (negative: no entry), logits bf16 or fp32 [M, top]; temperature
        from 1e-4 to 1e4."""
        extra, top = self._teacher(index, logits, temperature)
        return self._call(_base.lib().mlp_distill, W, H, extra, top, ws, False, loss, row_loss, None, None, None)

    def distill_step(self, W, H, index, logits, ws, temperature: float = 1.0, loss=None, row_loss=None, dH=None,
                     dW=None, dtype=torch.float32):
        """distill() and its gradients: (dH [M, dim], dW [dim, vocab], loss)."""
        extra, top = self._teacher(index, logits, temperature)
        return self._call(_base.lib().mlp_distill, W, H, extra, top, ws, True, loss, row_loss, dH, dW, dtype)
