"""Operators of a worker's local training step: the entry points of include/adacgd_train.h on torch tensors.

They stand between and behind a model's matrix products: layer norm with the residual sum and dropout in front of it,
dropout, log-probabilities of given tokens, and the preference and policy losses with their gradients with respect to
the logits.  What a worker computes with them is a gradient X_i = grad f_i(x), which `AdaCGD.compress` takes.

Every output is a tensor of the caller's; the arithmetic is in the kernels of libadacgd.so and there is no other path.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional

from .binding import AdacgdError, load_library

TRAIN_SYMBOLS = [
    "adacgd_train_workspace_bytes", "adacgd_train_init", "adacgd_train_destroy", "adacgd_train_last_error",
    "adacgd_train_launch_count", "adacgd_dropout", "adacgd_layer_norm", "adacgd_layer_norm_backward",
    "adacgd_token_logp", "adacgd_preference_loss", "adacgd_policy_loss",
]
MAX_COLS = 32768
PREFERENCE_KINDS = {"sigmoid": 0, "hinge": 1, "square": 2}

_vp, _i32, _i64, _u64, _f32, _f64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_float, C.c_double
_DROP = [("p", _f64), ("seed", _u64), ("offset", _u64)]


def _matrix(name):
    return [(name, _vp), (name + "_stride", _i64)]


class _DropoutArgs(C.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), *_matrix("x"), *_matrix("residual"), *_matrix("out"), ("dtype", _i32),
                ("reserved", _i32), *_DROP]


class _NormArgs(C.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), *_matrix("x"), *_matrix("residual"), *_matrix("out"), *_matrix("sum"),
                ("weight", _vp), ("bias", _vp), ("mean", _vp), ("rstd", _vp), ("dtype", _i32), ("param_dtype", _i32),
                ("eps", _f32), ("reserved", _i32), *_DROP]


class _NormBackwardArgs(C.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), *_matrix("dout"), *_matrix("s"), *_matrix("dsum"), *_matrix("dx"),
                *_matrix("dresidual"), ("mean", _vp), ("rstd", _vp), ("weight", _vp), ("dweight", _vp), ("dbias", _vp),
                ("dtype", _i32), ("param_dtype", _i32), *_DROP]


_ROWS = [("tokens", _i64), ("vocab", _i64), *_matrix("logits"), ("labels", _vp), ("mask", _vp), ("seq_start", _vp),
         ("sequences", _i64), ("dtype", _i32), ("label_bytes", _i32)]


class _TokenRows(C.Structure):
    _fields_ = _ROWS


class _PreferenceArgs(C.Structure):
    _fields_ = _ROWS + [("ref_logp", _vp), *_matrix("dlogits"), ("loss", _vp), ("margin", _vp), ("seq_logp", _vp),
                        ("beta", _f32), ("label_smoothing", _f32), ("grad_scale", _f32), ("kind", _i32),
                        ("length_normalized", _i32), ("reserved", _i32)]


class _PolicyArgs(C.Structure):
    _fields_ = _ROWS + [("old_logp", _vp), ("advantages", _vp), ("ref_logp", _vp), *_matrix("dlogits"), ("loss", _vp),
                        ("logp", _vp), ("stats", _vp), ("clip_low", _f32), ("clip_high", _f32), ("kl_beta", _f32),
                        ("grad_scale", _f32), ("per_sequence", _i32), ("reserved", _i32)]


_bound = False


def load_training_library():
    """Loads libadacgd.so with the signatures of adacgd_train.h; raises if it has not been built."""
    global _bound
    lib = load_library()
    if not _bound:
        lib.adacgd_train_workspace_bytes.argtypes = [_i64, _i64, C.POINTER(C.c_size_t)]
        lib.adacgd_train_init.argtypes = [C.POINTER(_vp), _i64, _i64, _vp, C.c_size_t, _vp]
        lib.adacgd_train_destroy.argtypes = [_vp]
        lib.adacgd_train_destroy.restype = None
        lib.adacgd_train_last_error.argtypes = [_vp]
        lib.adacgd_train_last_error.restype = C.c_char_p
        lib.adacgd_train_launch_count.argtypes = [_vp]
        lib.adacgd_train_launch_count.restype = _i64
        for name, args in (("adacgd_dropout", _DropoutArgs), ("adacgd_layer_norm", _NormArgs),
                           ("adacgd_layer_norm_backward", _NormBackwardArgs), ("adacgd_preference_loss", _PreferenceArgs),
                           ("adacgd_policy_loss", _PolicyArgs)):
            getattr(lib, name).argtypes = [_vp, C.POINTER(args)]
        lib.adacgd_token_logp.argtypes = [_vp, C.POINTER(_TokenRows), _vp, _vp]
        _bound = True
    return lib


class TrainingOps:
    """Owns a context of the training operators and the device workspace behind it.

    max_tokens bounds the rows of a norm's backward pass and of logits, max_cols the columns of a norm's backward pass.
    Work runs on `stream` (default: the stream that is current now).  A call made while another stream is current is
    ordered behind that stream's work, and that stream waits for it.  One thread at a time per context.

    Matrices are 2-D with unit column stride and any row stride, of type float32, float16 or bfloat16; vectors are
    contiguous.  Outputs may be the very same tensor as an input matrix of the same call (in place)."""

    def __init__(self, max_tokens: int, max_cols: int = 8192, *, device="cuda:0", stream=None):
        import torch

        self.torch = torch
        self.lib = load_training_library()
        if not torch.cuda.is_available():
            raise RuntimeError("the training operators need a CUDA device; there is no CPU path")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.index = self.device.index
        self.max_tokens, self.max_cols = int(max_tokens), int(max_cols)
        self._types = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
        self._f32, self._u8, self._bool = torch.float32, torch.uint8, torch.bool
        self._i64, self._i32 = torch.int64, torch.int32
        self.ctx = None
        nbytes = C.c_size_t(0)
        self._check(self.lib.adacgd_train_workspace_bytes(self.max_tokens, self.max_cols, C.byref(nbytes)), None)
        with torch.cuda.device(self.index):
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
            with torch.cuda.stream(self.stream):   # the workspace belongs to the stream that uses it
                self.workspace = torch.empty(nbytes.value + 256, dtype=torch.uint8, device=self.device)
            base = (self.workspace.data_ptr() + 255) // 256 * 256
            ctx = C.c_void_p()
            self._check(self.lib.adacgd_train_init(C.byref(ctx), self.max_tokens, self.max_cols, C.c_void_p(base), nbytes.value,
                                                   C.c_void_p(self.stream.cuda_stream)), None)
        self.ctx = ctx
        self.workspace_bytes = nbytes.value

    # -- helpers ---------------------------------------------------------
    def _check(self, status: int, ctx):
        if status != 0:
            raise AdacgdError(status, self.lib.adacgd_train_last_error(ctx).decode())

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.adacgd_train_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _call(self, entry, *args):
        """The entry point on the context's device, in the order of the current stream."""
        cuda = self.torch.cuda
        if self.ctx is None:
            raise RuntimeError("the context is closed")
        if cuda.current_device() != self.index:
            with cuda.device(self.index):
                return self._call(entry, *args)
        current = cuda.current_stream(self.index)
        if current.cuda_stream == self.stream.cuda_stream:
            status = entry(self.ctx, *args)
        else:
            self.stream.wait_stream(current)
            status = entry(self.ctx, *args)
            current.wait_stream(self.stream)
        if status != 0:
            self._check(status, self.ctx)

    def _mat(self, t, shape, dtype, name):
        """(pointer, row stride) of a matrix argument."""
        if t is None:
            return None, 0
        if t.dtype is not dtype or t.get_device() != self.index:
            raise ValueError(f"{name} must be a {dtype} tensor on {self.device}")
        if t.shape != shape:
            raise ValueError(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
        row, col = t.stride()
        if col != 1 and shape[1] > 1:
            raise ValueError(f"{name} must have unit column stride")
        if row < shape[1]:
            if shape[0] > 1:
                raise ValueError(f"{name}: rows overlap (stride {row} for {shape[1]} columns)")
            row = shape[1]
        return t.data_ptr(), row

    def _vec(self, t, n, dtype, name):
        """Pointer of a contiguous vector argument."""
        if t is None:
            return None
        if t.dtype is not dtype or t.get_device() != self.index:
            raise ValueError(f"{name} must be a {dtype} tensor on {self.device}")
        if t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous with {n} elements")
        return t.data_ptr()

    def _type(self, t, name):
        code = self._types.get(t.dtype)
        if code is None or t.dim() != 2:
            raise ValueError(f"{name} must be a 2-D float32, float16 or bfloat16 tensor")
        return code

    def _params(self, dtype, cols, **tensors):
        """(param type code, pointers) of weight-like vectors: all of the activations' type or all float32."""
        param = None
        for name, t in tensors.items():
            if t is not None:
                if param is None:
                    param = t.dtype
                    if param is not dtype and param is not self._f32:
                        raise ValueError(f"{name} must be {dtype} or float32")
                elif t.dtype is not param:
                    raise ValueError("weight-like arguments must share one type")
        return self._types[param or dtype], [self._vec(t, cols, param, name) for name, t in tensors.items()]

    def _rows(self, logits, labels, mask, seq_start, sequences):
        """Fields of adacgd_token_rows."""
        code = self._type(logits, "logits")
        shape = logits.shape
        n = shape[0]
        ptr, stride = self._mat(logits, shape, logits.dtype, "logits")
        ldt = labels.dtype
        if ldt is not self._i64 and ldt is not self._i32:
            raise ValueError("labels must be int64 or int32")
        if mask is not None and mask.dtype is not self._bool and mask.dtype is not self._u8:
            raise ValueError("mask must be bool or uint8")
        if seq_start is not None:
            if sequences is not None and sequences != seq_start.numel() - 1:
                raise ValueError("sequences and seq_start disagree")
            sequences = seq_start.numel() - 1
        return (n, shape[1], ptr, stride, self._vec(labels, n, ldt, "labels"),
                self._vec(mask, n, mask.dtype if mask is not None else None, "mask"),
                self._vec(seq_start, sequences + 1 if seq_start is not None else 0, self._i32, "seq_start"),
                sequences if sequences is not None else 1, code, 8 if ldt is self._i64 else 4)

    # -- entry points ------------------------------------------------------
    def dropout(self, x, out, *, p: float, seed: int, offset: int = 0, residual=None):
        """adacgd_dropout: out = [residual +] dropout(x).  The backward pass is the same call on the gradient."""
        code, shape, dt = self._type(x, "x"), x.shape, x.dtype
        a = _DropoutArgs(shape[0], shape[1], *self._mat(x, shape, dt, "x"), *self._mat(residual, shape, dt, "residual"),
                         *self._mat(out, shape, dt, "out"), code, 0, p, seed, offset)
        self._call(self.lib.adacgd_dropout, C.byref(a))

    def layer_norm(self, x, out, *, weight=None, bias=None, eps: float = 1e-5, residual=None, sum_out=None, mean=None,
                   rstd=None, p: float = 0.0, seed: int = 0, offset: int = 0):
        """adacgd_layer_norm: out = norm(s) with s = [residual +] dropout(x); sum_out receives s, mean and rstd the rows'
        statistics (float32), which the backward pass needs."""
        code, shape, dt = self._type(x, "x"), x.shape, x.dtype
        rows, cols = shape
        pcode, (w, b) = self._params(dt, cols, weight=weight, bias=bias)
        a = _NormArgs(rows, cols, *self._mat(x, shape, dt, "x"), *self._mat(residual, shape, dt, "residual"),
                      *self._mat(out, shape, dt, "out"), *self._mat(sum_out, shape, dt, "sum_out"), w, b,
                      self._vec(mean, rows, self._f32, "mean"), self._vec(rstd, rows, self._f32, "rstd"), code, pcode, eps, 0,
                      p, seed, offset)
        self._call(self.lib.adacgd_layer_norm, C.byref(a))

    def layer_norm_backward(self, dout, s, mean, rstd, dx, *, weight=None, dweight=None, dbias=None, dsum=None,
                            dresidual=None, p: float = 0.0, seed: int = 0, offset: int = 0):
        """adacgd_layer_norm_backward: dx, and where given dresidual, dweight, dbias, from dout and what layer_norm stored;
        dsum is the gradient that reaches s from elsewhere."""
        code, shape, dt = self._type(dout, "dout"), dout.shape, dout.dtype
        rows, cols = shape
        pcode, (w, dw, db) = self._params(dt, cols, weight=weight, dweight=dweight, dbias=dbias)
        a = _NormBackwardArgs(rows, cols, *self._mat(dout, shape, dt, "dout"), *self._mat(s, shape, dt, "s"),
                              *self._mat(dsum, shape, dt, "dsum"), *self._mat(dx, shape, dt, "dx"),
                              *self._mat(dresidual, shape, dt, "dresidual"), self._vec(mean, rows, self._f32, "mean"),
                              self._vec(rstd, rows, self._f32, "rstd"), w, dw, db, code, pcode, p, seed, offset)
        self._call(self.lib.adacgd_layer_norm_backward, C.byref(a))

    def token_logp(self, logits, labels, logp, *, mask=None, lse=None):
        """adacgd_token_logp: logp[t] = log softmax(logits[t])[labels[t]] where the mask is true, else 0."""
        rows = self._rows(logits, labels, mask, None, None)
        a = _TokenRows(*rows)
        self._call(self.lib.adacgd_token_logp, C.byref(a), self._vec(logp, rows[0], self._f32, "logp"),
                   self._vec(lse, rows[0], self._f32, "lse"))

    def preference_loss(self, logits, labels, ref_logp, loss, dlogits=None, *, mask=None, sequences: Optional[int] = None,
                        seq_start=None, beta: float = 0.1, kind: str = "sigmoid", label_smoothing: float = 0.0,
                        length_normalized: bool = False, grad_scale: float = 1.0, margin=None, seq_logp=None):
        """adacgd_preference_loss over pairs of sequences: the first half of them preferred, the second half rejected.
        Sequences are `sequences` equal runs of rows, or the runs that seq_start (int32, on the device) gives."""
        if sequences is None and seq_start is None:
            raise ValueError("preference_loss needs sequences or seq_start")
        if kind not in PREFERENCE_KINDS:
            raise ValueError(f"unknown kind {kind!r}; one of {tuple(PREFERENCE_KINDS)}")
        rows = self._rows(logits, labels, mask, seq_start, sequences)
        n, q, f32 = rows[0], rows[7], self._f32
        a = _PreferenceArgs(*rows, self._vec(ref_logp, n, f32, "ref_logp"),
                            *self._mat(dlogits, logits.shape, logits.dtype, "dlogits"), self._vec(loss, 1, f32, "loss"),
                            self._vec(margin, q // 2, f32, "margin"), self._vec(seq_logp, q, f32, "seq_logp"), beta,
                            label_smoothing, grad_scale, PREFERENCE_KINDS[kind], 1 if length_normalized else 0, 0)
        self._call(self.lib.adacgd_preference_loss, C.byref(a))

    def policy_loss(self, logits, labels, old_logp, advantages, loss, dlogits=None, *, mask=None,
                    sequences: Optional[int] = None, seq_start=None, ref_logp=None, clip_low: float = 0.2,
                    clip_high: float = 0.2, kl_beta: float = 0.0, per_sequence: bool = False, grad_scale: float = 1.0,
                    logp=None, stats=None):
        """adacgd_policy_loss: the clipped policy loss with a KL term, a mean over counted tokens or (per_sequence) over
        sequences of the mean over their counted tokens.  advantages: one float32 a token."""
        if per_sequence and sequences is None and seq_start is None:
            raise ValueError("per_sequence needs sequences or seq_start")
        rows = self._rows(logits, labels, mask, seq_start, sequences)
        n, f32 = rows[0], self._f32
        a = _PolicyArgs(*rows, self._vec(old_logp, n, f32, "old_logp"), self._vec(advantages, n, f32, "advantages"),
                        self._vec(ref_logp, n, f32, "ref_logp"), *self._mat(dlogits, logits.shape, logits.dtype, "dlogits"),
                        self._vec(loss, 1, f32, "loss"), self._vec(logp, n, f32, "logp"), self._vec(stats, 3, f32, "stats"),
                        clip_low, clip_high, kl_beta, grad_scale, 1 if per_sequence else 0, 0)
        self._call(self.lib.adacgd_policy_loss, C.byref(a))

    def launch_count(self) -> int:
        return int(self.lib.adacgd_train_launch_count(self.ctx))
