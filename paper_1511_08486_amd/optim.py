"""AdamW over many tensors at once and the norm of many gradients, over the sfb_adamw_* and sfb_grad_norm entry points.
Marshalling only, like the rest of the binding: the tensors' tables are made once, a step is one call."""
from __future__ import annotations

import ctypes as C

import torch

from .binding import SFB_BF16, SFB_F32, SFB_MLR, SfbError, lib, sfb_adamw, sfb_adamw_tensor, sfb_gradient


class _Stream:
    """An sfb_ctx that carries a stream for calls that need nothing else of it."""

    def __init__(self, stream, device, shape=(SFB_MLR, 1, 1, 1, 1, SFB_F32)):
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device(self.device.type, torch.cuda.current_device())
        if stream is None:
            stream = torch.cuda.current_stream(self.device).cuda_stream
        self.stream = int(stream)
        self._ctx = C.c_void_p()
        with torch.cuda.device(self.device):
            self._check(lib.sfb_create(C.byref(self._ctx), *shape, C.c_void_p(self.stream)), "sfb_create")

    def _scratch(self, nbytes):
        """A workspace that is this stream's own from the allocator on.  (From the current stream's memory it could be a block that was freed
        there while what used it still waits to run.)"""
        with torch.cuda.stream(torch.cuda.ExternalStream(self.stream, device=self.device)):
            return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=self.device)

    def _check(self, status, where):
        if status != 0:
            raise SfbError(status, where, lib.sfb_last_hip_error(self._ctx) if self._ctx else 0)

    def sync(self):
        self._check(lib.sfb_sync(self._ctx), "sfb_sync")

    def close(self):
        if getattr(self, "_ctx", None):
            lib.sfb_destroy(self._ctx)
            self._ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _dense(ts, what, device, dtypes, like=None):
    """Checks a list of dense tensors of one type; with `like`, of the same lengths."""
    ts = list(ts)
    if like is not None and len(ts) != len(like):
        raise ValueError(f"{what}: {len(ts)} tensors for {len(like)}")
    for i, t in enumerate(ts):
        if t.device != device or t.dtype not in dtypes or t.dtype != ts[0].dtype or not t.is_contiguous():
            raise ValueError(f"{what}[{i}]: wants a dense tensor of one of {dtypes} on {device}, all of one type")
        if like is not None and t.numel() != like[i]:
            raise ValueError(f"{what}[{i}]: {t.numel()} elements for {like[i]}")
    return ts


def _one(t, what, device, dtype, n=1):
    if t is None:
        return None
    if t.device != device or t.dtype != dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError(f"{what}: wants {n} {dtype} on {device}")
    return t.data_ptr()


_GRADS = (torch.float32, torch.bfloat16)


class GradNorm(_Stream):
    """The norm of `grads` (fp32 or bf16, all of one type) as one vector, and the factor that clips it:
    out[0] = norm, out[1] = min(1, max_norm / norm), NaN if the norm is not finite.  Both stay on the device; hand out[1:] to
    AdamW.step as grad_scale.  The gradients' memory is that of the construction; `grads` are kept alive with the object.  Calls that may
    overlap in time, replays of captured ones included, need an object each (it holds a workspace).  Calls run on `stream`, the one
    that was current at construction by default; work of other streams on the same tensors is ordered by the caller."""

    def __init__(self, grads, stream=None, device="cuda:0"):
        super().__init__(stream, device)
        self.grads = _dense(grads, "grads", self.device, _GRADS)
        self._list = (sfb_gradient * max(1, len(self.grads)))(*[sfb_gradient(t.data_ptr(), t.numel()) for t in self.grads])
        need = C.c_size_t()
        self._check(lib.sfb_grad_norm_bytes(self._list, len(self.grads), C.byref(need)), "sfb_grad_norm_bytes")
        self._ws = self._scratch(need.value)
        self._dtype = SFB_BF16 if self.grads and self.grads[0].dtype == torch.bfloat16 else SFB_F32

    def __call__(self, max_norm, out):
        self._check(lib.sfb_grad_norm(self._ctx, self._list, len(self.grads), self._dtype, float(max_norm),
                                      _one(out, "out", self.device, torch.float32, 2), self._ws.data_ptr(), self._ws.numel()),
                    "sfb_grad_norm")
        return out


class AdamW(_Stream):
    """AdamW over lists of tensors: params fp32, grads fp32 or bf16, first and second moments fp32 or, with m_scales and v_scales
    (uint8, one for every 128 elements), uint8 codes; copies: bf16 tensors that receive the rounded parameters, or None.
    `step` is a device int32 that holds the steps taken (0 at first) and goes on counting in a replayed graph.  8-bit moments start
    as zeros.  All tensors are kept alive with the object and keep their memory; step(grads=...) takes others from then on.
    Steps run on `stream`, the one that was current at construction by default.  Work of other streams on the same tensors is ordered
    by the caller, who keeps replaced gradients, and an object that is dropped, until the stream is through with them."""

    def __init__(self, params, grads, m, v, step, m_scales=None, v_scales=None, copies=None, stream=None, device="cuda:0"):
        super().__init__(stream, device)
        dev = self.device
        self.params = _dense(params, "params", dev, (torch.float32,))
        n = self.sizes = [t.numel() for t in self.params]
        if (m_scales is None) != (v_scales is None):
            raise ValueError("m_scales and v_scales come together")
        self.bits = 32 if m_scales is None else 8
        state = (torch.float32,) if self.bits == 32 else (torch.uint8,)
        self.m, self.v = _dense(m, "m", dev, state, n), _dense(v, "v", dev, state, n)
        blocks = [(k + 127) // 128 for k in n]
        self.m_scales = _dense(m_scales, "m_scales", dev, (torch.uint8,), blocks) if m_scales is not None else [None] * len(n)
        self.v_scales = _dense(v_scales, "v_scales", dev, (torch.uint8,), blocks) if v_scales is not None else [None] * len(n)
        self.copies = _dense(copies, "copies", dev, (torch.bfloat16,), n) if copies is not None else [None] * len(n)
        self.taken = step
        self._step = _one(step, "step", dev, torch.int32)
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self._list = (sfb_adamw_tensor * max(1, len(n)))(*[
            sfb_adamw_tensor(ptr(p), None, ptr(a), ptr(b), ptr(c), ptr(d), ptr(e), k) for p, a, b, c, d, e, k in
            zip(self.params, self.m, self.v, self.m_scales, self.v_scales, self.copies, n)])
        self._bind(grads)

    def _bind(self, grads):
        self.grads = _dense(grads, "grads", self.device, _GRADS, self.sizes)
        for entry, t in zip(self._list, self.grads):
            entry.g = t.data_ptr()
        self._grad_dtype = SFB_BF16 if self.grads and self.grads[0].dtype == torch.bfloat16 else SFB_F32

    def step(self, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, seed=0, grad_scale=None, lr_scale=None, grads=None):
        if grads is not None:
            self._bind(grads)
        o = sfb_adamw(float(lr), float(betas[0]), float(betas[1]), float(eps), float(weight_decay), self.bits, self._grad_dtype,
                      int(seed) & 0xFFFFFFFF, self._step, _one(grad_scale, "grad_scale", self.device, torch.float32),
                      _one(lr_scale, "lr_scale", self.device, torch.float32))
        self._check(lib.sfb_adamw_step(self._ctx, self._list, len(self.sizes), C.byref(o)), "sfb_adamw_step")

    def unpack(self, m_out, v_out):
        """The values of 8-bit moments, exactly, into bf16 tensors."""
        if self.bits != 8:
            raise ValueError("the moments are fp32")
        outs = [_dense(x, w, self.device, (torch.bfloat16,), self.sizes) for x, w in ((m_out, "m_out"), (v_out, "v_out"))]
        arrays = [(C.c_void_p * max(1, len(x)))(*[t.data_ptr() for t in x]) for x in outs]
        self._check(lib.sfb_adamw_unpack(self._ctx, self._list, len(self.sizes), *arrays), "sfb_adamw_unpack")
