"""The output layer of a model: softmax cross entropy of a linear head over a large vocabulary, with the gradients by the features and
by W, without the scores in memory (the sfb_xent_* entry points).  Marshalling only."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import SFB_BF16, SFB_F32, SFB_MLR, lib, sfb_xent
from .optim import _Stream, _one

_DTYPES = {"f32": (SFB_F32, torch.float32), "bf16": (SFB_BF16, torch.bfloat16)}


class SoftmaxHead(_Stream):
    """A head of J words on D features for up to `rows` rows a call, features in `dtype`, W in `w_dtype` ("f32" or "bf16").
    Owns an sfb_ctx and a workspace (workspace_bytes: as many, at least what the calls need; default: as many as speed them up).
    Rows whose label is outside [0, J) take no part.  Gradients come in the types of the features and of W; give one or both.
    `gradients` reads the lse that `loss` left; `loss_and_gradients` is both in one call.  Calls that may overlap in time, replays of
    captured ones included, need a head each (it holds a workspace).
    Calls run on `stream`, the one that was current at construction by default, whichever is current when they are made.  Work of other
    streams on the same tensors is ordered by the caller, who also keeps them until the call has run."""

    def __init__(self, J, D, rows, dtype="bf16", w_dtype="bf16", workspace_bytes=None, gradients=True, stream=None, device="cuda:0"):
        self._a, self._w = _DTYPES[dtype], _DTYPES[w_dtype]
        self.J, self.D, self.rows = int(J), int(D), int(rows)
        super().__init__(stream, device, (SFB_MLR, self.J, self.D, 1, self.rows, self._a[0]))
        least, best = C.c_size_t(), C.c_size_t()
        self._check(lib.sfb_xent_workspace_bytes(self._ctx, self._w[0], 1 if gradients else 0, C.byref(least), C.byref(best)),
                    "sfb_xent_workspace_bytes")
        self.least_bytes, self.best_bytes = least.value, best.value
        self._ws = self._scratch(self.best_bytes if workspace_bytes is None else workspace_bytes)

    def _matrix(self, t, what, rows, dtype):
        if t is None:
            return None, 0
        if t.device != self.device or t.dtype != dtype or t.dim() != 2 or tuple(t.shape) != (rows, self.D) or (t.stride(1) != 1 and self.D > 1):
            raise ValueError(f"{what}: wants [{rows}, {self.D}] {dtype} on {self.device}, dense along its rows")
        return t.data_ptr(), (t.stride(0) if rows > 1 else max(t.stride(0), self.D))

    def _call(self, name, W, a, y, loss, lse, total, weight, dA, dW, scale, mean):
        n, dev, f = int(a.shape[0]), self.device, torch.float32
        x = sfb_xent()
        x.W, x.ldw = self._matrix(W, "W", self.J, self._w[1])
        x.w_dtype, x.mean, x.n, x.scale = self._w[0], 1 if mean else 0, n, float(scale)
        x.a, x.lda = self._matrix(a, "a", n, self._a[1])
        x.y = _one(y, "y", dev, torch.int32, n)
        x.loss, x.lse = _one(loss, "loss", dev, f, n), _one(lse, "lse", dev, f, n)
        x.total, x.weight = _one(total, "total", dev, f), _one(weight, "weight", dev, f, n)
        x.dA, x.ldda = self._matrix(dA, "dA", n, self._a[1])
        x.dW, x.lddw = self._matrix(dW, "dW", self.J, self._w[1])
        x.ws, x.ws_bytes = self._ws.data_ptr(), self._ws.numel()
        self._check(getattr(lib, name)(self._ctx, C.byref(x)), name)

    def loss(self, W, a, y, loss=None, lse=None, total=None, weight=None, scale=1.0, mean=False):
        self._call("sfb_xent_loss", W, a, y, loss, lse, total, weight, None, None, scale, mean)

    def gradients(self, W, a, y, lse, dA=None, dW=None, weight=None, scale=1.0, mean=False):
        self._call("sfb_xent_gradients", W, a, y, None, lse, None, weight, dA, dW, scale, mean)

    def loss_and_gradients(self, W, a, y, loss=None, lse=None, dA=None, dW=None, total=None, weight=None, scale=1.0, mean=False):
        self._call("sfb_xent_loss_and_gradients", W, a, y, loss, lse, total, weight, dA, dW, scale, mean)
