"""The operators of networks whose layers are Kronecker products, on torch CUDA tensors: layer norm, the gated feed-forward block
and the softmax cross entropy over a large vocabulary, each forward and backward.  Argument marshalling only, as in binding.py.

There is no autograd: results have no history, whatever their inputs require, and the gradients' functions are called by the training step itself
(examples/language_model.py is one).

Tensors are float32 or bfloat16, all of a call's alike (statistics, losses and their gradients are float32), 2-D and on one device.  In bfloat16 the
gradients of products have operands of one bfloat16 each and errors of 2.3e-3 to 2.9e-3 of their norm, where one rounding leaves 1.7e-3.  Rows of
X, dY and dH may lie further apart than they are long (a column range of a larger tensor); everything else is contiguous.
Products have two factors, (F1, F2) of P1 x Q1 and P2 x Q2 with P1, P2 up to 128: X has P1*P2 columns, X (F1 (x) F2) has Q1*Q2.

Every call is asynchronous on `stream` (a raw hipStream_t value; default: torch's current stream), on which its results and its
workspace are allocated too.  Inputs made on another stream are the caller's to wait for and to keep, as with any torch operation."""
import ctypes
import operator
from contextlib import nullcontext

from . import binding
from .binding import KM_ACT_GELU_TANH, KM_ACT_SILU, KM_BF16, KM_F32, _check, _current_stream, _entry

_ACTIVATIONS = {"silu": KM_ACT_SILU, "gelu_tanh": KM_ACT_GELU_TANH}
_Two, _Pointers = ctypes.c_int * 2, ctypes.c_void_p * 2


def _native():
    """The binding's native part: takes calls of plain tensors on the current stream with results of its own making.  What it declines
    goes the long way below, which also says what is wrong."""
    return binding._native or binding._start_native()


def _code(dtype):
    import torch
    if dtype is torch.bfloat16:
        return KM_BF16
    if dtype is torch.float32:
        return KM_F32
    raise TypeError("unsupported dtype %s (float32 and bfloat16 only)" % dtype)


def _rows(name, t, like=None, columns=None):
    """Checks a matrix whose rows may lie apart and returns the distance."""
    if not t.is_cuda or t.dim() != 2:
        raise ValueError("%s must be a 2-D CUDA tensor" % name)
    m, n = t.shape
    if like is not None and (t.dtype != like.dtype or t.get_device() != like.get_device() or m != like.shape[0]):
        raise ValueError("%s must have X's dtype, device and number of rows" % name)
    if columns is not None and n != columns:
        raise ValueError("%s has %d columns instead of %d" % (name, n, columns))
    if n > 1 and t.stride(1) != 1:
        raise ValueError("%s must have contiguous rows" % name)
    if m < 2:
        return n
    if t.stride(0) < n:
        raise ValueError("rows of %s overlap" % name)
    return t.stride(0)


def _vector(name, t, n, dtype, index):
    if t.get_device() != index or t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError("%s must be a contiguous CUDA tensor of %d elements of %s on X's device" % (name, n, dtype))


def _factors(name, fs, X, shapes=None):
    """Checks two factors; returns (P, Q, pointers) for C and the shapes."""
    if len(fs) != 2:
        raise ValueError("%s must be two factors" % name)
    index = X.get_device()
    for f in fs:
        if f.dim() != 2 or f.dtype != X.dtype or f.get_device() != index or not f.is_contiguous():
            raise ValueError("%s must be contiguous 2-D CUDA tensors of X's dtype and device" % name)
    a, b = fs
    found = (a.shape[0], a.shape[1], b.shape[0], b.shape[1])
    if shapes is not None and found != shapes:
        raise ValueError("the factors of %s have other shapes than those before them" % name)
    if X.shape[1] != found[0] * found[2]:
        raise ValueError("X has %d columns, %s needs %d" % (X.shape[1], name, found[0] * found[2]))
    return _Two(found[0], found[2]), _Two(found[1], found[3]), _Pointers(a.data_ptr(), b.data_ptr()), found


class _On:
    """Where a call runs: `with _On(X, stream) as raw_stream`."""

    def __init__(self, X, stream):
        import torch
        self.index, self.stream = X.get_device(), stream
        self.device = nullcontext() if torch.cuda.current_device() == self.index else torch.cuda.device(self.index)
        self.on = nullcontext()

    def __enter__(self):
        self.device.__enter__()
        if self.stream is None:
            return _current_stream(self.index)
        import torch
        self.on = torch.cuda.stream(torch.cuda.ExternalStream(self.stream, device=self.index) if self.stream else torch.cuda.default_stream(self.index))
        self.on.__enter__()
        return self.stream

    def __exit__(self, *error):
        self.on.__exit__(*error)
        self.device.__exit__(*error)


def _bytes(name, *args):
    out = ctypes.c_size_t(0)
    name = "kronmatmul_" + name + "_workspace_size"
    _check(_entry(name)(*args, ctypes.byref(out)), name)
    return out.value


def _workspace(X, need):
    import torch
    return X.new_empty((need,), dtype=torch.uint8) if need else None


def _call(name, *args):
    name = "kronmatmul_" + name
    _check(_entry(name)(*args), name)


def layer_norm(X, weight, bias=None, eps=1e-5, Y=None, stream=None):
    """(X - mean) * rstd * weight + bias over the rows of X.  Returns (Y, mean, rstd), the latter two (one float32 per row) for
    layer_norm_grad.  Y: where the result goes (default: a new tensor)."""
    if stream is None and Y is None:
        got = _native().layer_norm(X, weight, bias, eps)
        if got is not NotImplemented:
            return got
    import torch
    ldx = _rows("X", X)
    (m, h), dtype, index, code = X.shape, X.dtype, X.get_device(), _code(X.dtype)
    if h < 1:
        raise ValueError("X has no columns")
    _vector("weight", weight, h, dtype, index)
    if bias is not None:
        _vector("bias", bias, h, dtype, index)
    with _On(X, stream) as s:
        if Y is None:
            Y = X.new_empty((m, h))
        elif Y.dtype != dtype or Y.get_device() != index or Y.shape != X.shape or not Y.is_contiguous():
            raise ValueError("Y must be a contiguous CUDA tensor of shape (%d, %d)" % (m, h))
        stats = X.new_empty((2, m), dtype=torch.float32)
        mean, rstd = stats.unbind()
        if m:
            _call("layer_norm", m, h, X.data_ptr(), ldx, weight.data_ptr(), bias.data_ptr() if bias is not None else None, eps, Y.data_ptr(),
                  mean.data_ptr(), rstd.data_ptr(), code, s)
    return Y, mean, rstd


def layer_norm_grad(dY, X, weight, mean, rstd, bias=True, stream=None):
    """(dX, dweight, dbias) from the gradient of layer_norm's Y and what went into and came out of that call.  bias=False: the norm had none,
    dbias is None."""
    if stream is None:
        got = _native().layer_norm_grad(dY, X, weight, mean, rstd, bias)
        if got is not NotImplemented:
            return got
    import torch
    ldx = _rows("X", X)
    (m, h), index, code = X.shape, X.get_device(), _code(X.dtype)
    if h < 1:
        raise ValueError("X has no columns")
    lddy = _rows("dY", dY, X, h)
    _vector("weight", weight, h, X.dtype, index)
    _vector("mean", mean, m, torch.float32, index)
    _vector("rstd", rstd, m, torch.float32, index)
    with _On(X, stream) as s:
        dX, dw = X.new_empty((m, h)), X.new_empty((h,))
        db = X.new_empty((h,)) if bias else None
        if not m:
            return dX, dw.zero_(), db.zero_() if bias else None
        need = _bytes("layer_norm_grad", m, h, code)
        ws = _workspace(X, need)
        _call("layer_norm_grad", m, h, dY.data_ptr(), lddy, X.data_ptr(), ldx, weight.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dX.data_ptr(),
              dw.data_ptr(), db.data_ptr() if bias else None, code, ws.data_ptr() if need else None, need, s)
    return dX, dw, db


def _activation(act):
    code = _ACTIVATIONS.get(act)
    if code is None:
        raise ValueError("act must be one of %s" % ", ".join(_ACTIVATIONS))
    return code


def kron_gated(X, gate, up, act="silu", H=None, stream=None):
    """The gated feed-forward block's inner activations, act(X (gate[0] (x) gate[1])) * (X (up[0] (x) up[1])), in one kernel.  act: "silu"
    or "gelu_tanh".  H: where the result goes (default: a new tensor).  A projection back is a kronmatmul of H, in float32 only, and for its factors there is no
    gradient here."""
    if stream is None and H is None:
        got = _native().gated(X, gate, up, _activation(act))
        if got is not NotImplemented:
            return got
    code, act = _code(X.dtype), _activation(act)
    ldx = _rows("X", X)
    P, Q, pg, shapes = _factors("gate", gate, X)
    pu = _factors("up", up, X, shapes)[2]
    m, n = X.shape[0], shapes[1] * shapes[3]
    with _On(X, stream) as s:
        if H is None:
            H = X.new_empty((m, n))
        elif H.dtype != X.dtype or H.get_device() != X.get_device() or H.shape != (m, n) or not H.is_contiguous():
            raise ValueError("H must be a contiguous CUDA tensor of shape (%d, %d)" % (m, n))
        if m:
            _call("gated", m, P, Q, X.data_ptr(), ldx, pg, pu, act, H.data_ptr(), code, s)
    return H


def kron_gated_grad(dH, X, gate, up, act="silu", stream=None):
    """(dX, (dgate[0], dgate[1]), (dup[0], dup[1])) from the gradient of kron_gated's result and that call's arguments."""
    if stream is None:
        got = _native().gated_grad(dH, X, gate, up, _activation(act))
        if got is not NotImplemented:
            return got
    code, act = _code(X.dtype), _activation(act)
    ldx = _rows("X", X)
    P, Q, pg, shapes = _factors("gate", gate, X)
    pu = _factors("up", up, X, shapes)[2]
    m = X.shape[0]
    lddh = _rows("dH", dH, X, shapes[1] * shapes[3])
    with _On(X, stream) as s:
        dX = X.new_empty((m, X.shape[1]))
        dg, du = tuple(f.new_empty(f.shape) for f in gate), tuple(f.new_empty(f.shape) for f in up)
        if not m:
            return dX, tuple(f.zero_() for f in dg), tuple(f.zero_() for f in du)
        need = _bytes("gated_grad", m, P, Q, code)
        ws = _workspace(X, need)
        _call("gated_grad", m, P, Q, dH.data_ptr(), lddh, X.data_ptr(), ldx, pg, pu, act, dX.data_ptr(), _Pointers(dg[0].data_ptr(), dg[1].data_ptr()),
              _Pointers(du[0].data_ptr(), du[1].data_ptr()), code, ws.data_ptr() if need else None, need, s)
    return dX, dg, du


def _loss_arguments(X, Fs, targets, vocab):
    import torch
    code, ldx = _code(X.dtype), _rows("X", X)
    P, Q, pf, shapes = _factors("Fs", Fs, X)
    _vector("targets", targets, X.shape[0], torch.int64, X.get_device())
    columns = shapes[1] * shapes[3]
    vocab = columns if vocab is None else operator.index(vocab)
    if not 1 <= vocab <= columns:
        raise ValueError("vocab must be 1 to %d" % columns)
    return code, ldx, P, Q, pf, vocab


def kron_cross_entropy(X, Fs, targets, vocab=None, stream=None):
    """Softmax cross entropy of the logits X (Fs[0] (x) Fs[1]) without ever writing them.  Returns (loss, lse), float32 per token: the
    loss and the logarithm of the sum of the exponentials, which kron_cross_entropy_grad takes.  targets: int64 column numbers; a token whose
    target is not in 0..vocab-1 has a loss of 0.  vocab: how many columns of the product are words (default: all)."""
    if stream is None:
        got = _native().cross_entropy(X, Fs, targets, vocab)
        if got is not NotImplemented:
            return got
    import torch
    code, ldx, P, Q, pf, vocab = _loss_arguments(X, Fs, targets, vocab)
    m = X.shape[0]
    with _On(X, stream) as s:
        out = X.new_empty((2, m), dtype=torch.float32)
        loss, lse = out.unbind()
        if m:
            need = _bytes("cross_entropy", m, P, Q, vocab, code)
            ws = _workspace(X, need)
            _call("cross_entropy", m, P, Q, vocab, X.data_ptr(), ldx, pf, targets.data_ptr(), loss.data_ptr(), lse.data_ptr(), code,
                  ws.data_ptr() if need else None, need, s)
    return loss, lse


def kron_cross_entropy_grad(dloss, X, Fs, targets, lse, vocab=None, stream=None):
    """(dX, (dFs[0], dFs[1])) from dloss, the gradient of each token's loss (float32; 1/tokens for a mean), kron_cross_entropy's lse and that
    call's arguments.  Tokens without a target have no gradient, whatever their row of X holds."""
    if stream is None:
        got = _native().cross_entropy_grad(dloss, X, Fs, targets, lse, vocab)
        if got is not NotImplemented:
            return got
    import torch
    code, ldx, P, Q, pf, vocab = _loss_arguments(X, Fs, targets, vocab)
    m, index = X.shape[0], X.get_device()
    _vector("dloss", dloss, m, torch.float32, index)
    _vector("lse", lse, m, torch.float32, index)
    with _On(X, stream) as s:
        dX = X.new_empty((m, X.shape[1]))
        df = tuple(f.new_empty(f.shape) for f in Fs)
        if not m:
            return dX, tuple(f.zero_() for f in df)
        need = _bytes("cross_entropy_grad", m, P, Q, vocab, code)
        ws = _workspace(X, need)
        _call("cross_entropy_grad", m, P, Q, vocab, dloss.data_ptr(), X.data_ptr(), ldx, pf, targets.data_ptr(), lse.data_ptr(), dX.data_ptr(),
              _Pointers(df[0].data_ptr(), df[1].data_ptr()), code, ws.data_ptr() if need else None, need, s)
    return dX, df
