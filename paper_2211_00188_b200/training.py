"""Operators of a worker's local training step: the entry points of include/adacgd_train.h on torch tensors.

They stand between and behind a model's matrix products: embedding lookup, norm and rotation of queries and keys, attention,
each with its backward pass, layer norm with the residual sum and dropout in front of it, dropout, log-probabilities of given tokens, and the preference and policy losses with their gradients with respect to
the logits.  What a worker computes with them is a gradient X_i = grad f_i(x), which `AdaCGD.compress` takes.

Every output is a tensor of the caller's; the arithmetic is in the kernels of libadacgd.so and there is no other path.
The tensors are checked in a small extension module (csrc/adacgd_train_binding.cpp), because a small call would spend
most of its time on such checks in Python.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

from .binding import AdacgdError, load_library

TRAIN_SYMBOLS = [
    "adacgd_train_workspace_bytes", "adacgd_train_init", "adacgd_train_destroy", "adacgd_train_last_error",
    "adacgd_train_launch_count", "adacgd_dropout", "adacgd_layer_norm", "adacgd_layer_norm_backward",
    "adacgd_token_logp", "adacgd_preference_loss", "adacgd_policy_loss", "adacgd_embedding", "adacgd_embedding_backward",
    "adacgd_qk_norm", "adacgd_qk_norm_backward", "adacgd_attention", "adacgd_attention_backward",
]
MAX_COLS = 32768
PREFERENCE_KINDS = {"sigmoid": 0, "hinge": 1, "square": 2}
_RETRY = -1

_bound = False


def load_training_library():
    """Loads libadacgd.so with the signatures of adacgd_train.h; raises if it has not been built."""
    global _bound
    lib = load_library()
    if not _bound:
        vp, i64 = C.c_void_p, C.c_int64
        lib.adacgd_train_workspace_bytes.argtypes = [i64, i64, C.POINTER(C.c_size_t)]
        lib.adacgd_train_init.argtypes = [C.POINTER(vp), i64, i64, vp, C.c_size_t, vp]
        lib.adacgd_train_destroy.argtypes = [vp]
        lib.adacgd_train_destroy.restype = None
        lib.adacgd_train_last_error.argtypes = [vp]
        lib.adacgd_train_last_error.restype = C.c_char_p
        lib.adacgd_train_launch_count.argtypes = [vp]
        lib.adacgd_train_launch_count.restype = i64
        for name in ("adacgd_dropout", "adacgd_layer_norm", "adacgd_layer_norm_backward", "adacgd_preference_loss",
                     "adacgd_policy_loss", "adacgd_embedding", "adacgd_embedding_backward", "adacgd_qk_norm", "adacgd_qk_norm_backward",
                     "adacgd_attention", "adacgd_attention_backward"):
            getattr(lib, name).argtypes = [vp, vp]
        lib.adacgd_token_logp.argtypes = [vp, vp, vp, vp]
        _bound = True
    return lib


def _load_binding():
    import torch  # noqa: F401  (the module links against its libraries)

    from . import build

    if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_train_binding.so")):
        raise ImportError("_train_binding.so is missing: run `python -m paper_2211_00188_b200.build`")
    built_for = build.binding_built_for()
    if built_for not in (None, build.binding_target()):
        raise ImportError(f"_train_binding.so was built for {built_for}, this is {build.binding_target()}: run "
                          "`python -m paper_2211_00188_b200.build`")
    from . import _train_binding

    return _train_binding


class TrainingOps:
    """Owns a context of the training operators and the device workspace behind it.

    max_tokens bounds the rows of a norm's or lookup's backward pass and of logits, max_cols the columns of those backward passes.
    Work runs on `stream` (default: the stream that is current now).  A call made while another stream is current is
    ordered behind that stream's work, and that stream waits for it.  One thread at a time per context; graphs captured from
    one context are replayed one after the other.

    Matrices are 2-D with unit column stride and any row stride, of type float32, float16 or bfloat16; vectors are
    contiguous.  Rows must not overlap: an expanded row is refused.  Outputs may be the very same tensor as an input matrix
    of the same call (in place).  Wrong tensors raise ValueError, what the library refuses AdacgdError.

    The calls are outside autograd: they are not recorded, whether or not an input requires a gradient; the backward
    passes are the calls themselves.  An output that requires a gradient is refused while gradients are recorded, and
    what a call writes counts as modified in place, so a graph that has saved it says so when it runs backwards."""

    def __init__(self, max_tokens: int, max_cols: int = 8192, *, device="cuda:0", stream=None):
        import torch

        self.torch = torch
        self.lib = load_training_library()
        if not torch.cuda.is_available():
            raise RuntimeError("the training operators need a CUDA device; there is no CPU path")
        self.native = _load_binding()
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.index = self.device.index
        self.max_tokens, self.max_cols = int(max_tokens), int(max_cols)
        self.ctx = self.handle = None
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
        self.handle = self.native.bind(ctx.value, self.index, self.stream.cuda_stream)
        self.workspace_bytes = nbytes.value

    # -- helpers ---------------------------------------------------------
    def _check(self, status: int, ctx):
        if status != 0:
            raise AdacgdError(status, self.lib.adacgd_train_last_error(ctx).decode())

    def close(self):
        if getattr(self, "ctx", None):
            self.lib.adacgd_train_destroy(self.ctx)
            self.ctx = self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _again(self, status, function, *args):
        """What a call comes to that did not simply succeed: an error, or another current stream or device."""
        if status == _RETRY:
            cuda = self.torch.cuda
            with cuda.device(self.index):
                current = cuda.current_stream(self.index)
                if current.cuda_stream != self.stream.cuda_stream:
                    self.stream.wait_stream(current)
                self.native.force(self.handle, True)
                try:
                    status = function(*args)
                finally:
                    self.native.force(self.handle, False)
                if current.cuda_stream != self.stream.cuda_stream:
                    current.wait_stream(self.stream)
        self._check(status, self.ctx)

    # -- entry points ------------------------------------------------------
    def dropout(self, x, out, *, p: float, seed: int, offset: int = 0, residual=None):
        """adacgd_dropout: out = [residual +] dropout(x).  The backward pass is the same call on the gradient."""
        call, args = self.native.dropout, (self.handle, x, out, residual, p, seed, offset)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def layer_norm(self, x, out, *, weight=None, bias=None, eps: float = 1e-5, residual=None, sum_out=None, mean=None,
                   rstd=None, p: float = 0.0, seed: int = 0, offset: int = 0):
        """adacgd_layer_norm: out = norm(s) with s = [residual +] dropout(x); sum_out receives s, mean and rstd the rows'
        statistics (float32), which the backward pass needs."""
        call = self.native.layer_norm
        args = (self.handle, x, out, weight, bias, eps, residual, sum_out, mean, rstd, p, seed, offset)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def layer_norm_backward(self, dout, s, mean, rstd, dx, *, weight=None, dweight=None, dbias=None, dsum=None,
                            dresidual=None, p: float = 0.0, seed: int = 0, offset: int = 0):
        """adacgd_layer_norm_backward: dx, and where given dresidual, dweight, dbias, from dout and what layer_norm stored;
        dsum is the gradient that reaches s from elsewhere."""
        call = self.native.layer_norm_backward
        args = (self.handle, dout, s, mean, rstd, dx, weight, dweight, dbias, dsum, dresidual, p, seed, offset)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def token_logp(self, logits, labels, logp, *, mask=None, lse=None):
        """adacgd_token_logp: logp[t] = log softmax(logits[t])[labels[t]] where the mask is true, else 0."""
        call, args = self.native.token_logp, (self.handle, logits, labels, logp, mask, lse)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def preference_loss(self, logits, labels, ref_logp, loss, dlogits=None, *, mask=None, sequences: Optional[int] = None,
                        seq_start=None, beta: float = 0.1, kind: str = "sigmoid", label_smoothing: float = 0.0,
                        length_normalized: bool = False, grad_scale: float = 1.0, margin=None, seq_logp=None):
        """adacgd_preference_loss over pairs of sequences: the first half of them preferred, the second half rejected.
        Sequences are `sequences` equal runs of rows, or the runs that seq_start (int32, on the device) gives."""
        if sequences is None and seq_start is None:
            raise ValueError("preference_loss needs sequences or seq_start")
        if kind not in PREFERENCE_KINDS:
            raise ValueError(f"unknown kind {kind!r}; one of {tuple(PREFERENCE_KINDS)}")
        call = self.native.preference_loss
        args = (self.handle, logits, labels, ref_logp, loss, dlogits, mask, sequences, seq_start, beta, PREFERENCE_KINDS[kind],
                label_smoothing, length_normalized, grad_scale, margin, seq_logp)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def policy_loss(self, logits, labels, old_logp, advantages, loss, dlogits=None, *, mask=None,
                    sequences: Optional[int] = None, seq_start=None, ref_logp=None, clip_low: float = 0.2,
                    clip_high: float = 0.2, kl_beta: float = 0.0, per_sequence: bool = False, grad_scale: float = 1.0,
                    logp=None, stats=None):
        """adacgd_policy_loss: the clipped policy loss with a KL term, a mean over counted tokens or (per_sequence) over
        sequences of the mean over their counted tokens.  advantages: one float32 a token."""
        if per_sequence and sequences is None and seq_start is None:
            raise ValueError("per_sequence needs sequences or seq_start")
        call = self.native.policy_loss
        args = (self.handle, logits, labels, old_logp, advantages, loss, dlogits, mask, sequences, seq_start, ref_logp, clip_low,
                clip_high, kl_beta, per_sequence, grad_scale, logp, stats)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def embedding(self, tokens, table, out, *, scale: float = 1.0, mask=None):
        """adacgd_embedding: out[t] = scale * table[tokens[t]], 0 where the mask is false."""
        call, args = self.native.embedding, (self.handle, tokens, table, out, scale, mask)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def embedding_backward(self, tokens, dout, dtable, *, scale: float = 1.0, mask=None, base=None):
        """adacgd_embedding_backward: dtable = [base +] scale * sum of dout's rows by token, every row of it; dtable may be base
        itself.  dtable is of dout's type or float32."""
        call, args = self.native.embedding_backward, (self.handle, tokens, dout, dtable, scale, mask, base)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def qk_norm(self, q, k, q_out, k_out, positions=None, freq=None, *, head_dim: int, q_weight=None, k_weight=None, eps: float = 1e-6,
                interleaved: bool = False):
        """adacgd_qk_norm: every head of q and k divided by its root mean square, times the weight, its first 2 len(freq) elements
        turned by the angles position * freq (float32), in halves or, interleaved, in neighbours.  positions are int64 or int32; without
        freq there is no rotation.  k and k_out may be None."""
        call = self.native.qk_norm
        args = (self.handle, q, k, q_out, k_out, positions, freq, head_dim, q_weight, k_weight, eps, interleaved)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def qk_norm_backward(self, dq_out, dk_out, q, k, dq, dk, positions=None, freq=None, *, head_dim: int, q_weight=None, k_weight=None,
                         dq_weight=None, dk_weight=None, eps: float = 1e-6, interleaved: bool = False):
        """adacgd_qk_norm_backward: dq, dk and where given the weights' gradients, from the gradients of the outputs and the inputs
        of qk_norm."""
        call = self.native.qk_norm_backward
        args = (self.handle, dq_out, dk_out, q, k, dq, dk, positions, freq, head_dim, q_weight, k_weight, dq_weight, dk_weight, eps,
                interleaved)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def attention(self, q, k, v, out, *, heads: int, lse=None, sequences: Optional[int] = None, seq_start=None, causal: bool = True,
                  scale: Optional[float] = None, mask=None):
        """adacgd_attention over each sequence's tokens; scale defaults to head_dim ** -0.5.  k and v hold the key heads, whose number
        divides heads.  lse, float32 [heads, tokens], is what the backward pass needs.  Tokens where the mask is false are neither
        queries nor keys; their out is 0.  Rows of no sequence stay as they are.  No output may overlap anything."""
        if sequences is None and seq_start is None:
            raise ValueError("attention needs sequences or seq_start")
        call = self.native.attention
        args = (self.handle, q, k, v, out, lse, heads, sequences, seq_start, causal, scale, mask)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def attention_backward(self, dout, q, k, v, out, lse, row_dot, dq, dk, dv, *, heads: int, sequences: Optional[int] = None,
                           seq_start=None, causal: bool = True, scale: Optional[float] = None, mask=None):
        """adacgd_attention_backward: dq, dk and dv from dout and what attention took and stored.  row_dot, float32 [heads, tokens], is
        written on the way: the products of dout's and out's rows."""
        if sequences is None and seq_start is None:
            raise ValueError("attention_backward needs sequences or seq_start")
        call = self.native.attention_backward
        args = (self.handle, dout, q, k, v, out, lse, row_dot, dq, dk, dv, heads, sequences, seq_start, causal, scale, mask)
        status = call(*args)
        if status:
            self._again(status, call, *args)

    def launch_count(self) -> int:
        return int(self.lib.adacgd_train_launch_count(self.ctx))
