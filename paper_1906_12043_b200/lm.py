"""Thin binding over the language-model operators of libcocod.so (include/cocod_lm.h).

Marshalling only (csrc/lm_binding.cpp looks at the tensors and makes the calls): every product, sum and exponential is computed
by the library's CUDA kernels.  torch is used for device memory and streams.  No CPU fallback.

    ops = LMOps()
    y  = ops.grouped_forward(x, w, offsets)              # rows offsets[g] .. offsets[g + 1] - 1 times w[g]^T
    dx = ops.grouped_input_grad(dy, w, offsets)
    dw = ops.grouped_weight_grad(dy, x, offsets)         # x: a tensor or the PackedActivations of one
    kept = ops.act_pack(x)                               # 8 bits per value until the backward pass
    dz = ops.act_relu_grad(dh, kept)                     # dh where the kept activation is positive
    loss, row_loss, dx, dw = ops.vocab_loss_grad(x, w, labels, offsets)
"""
from __future__ import annotations

import ctypes

import torch

from . import engine as _E

BF16, F32 = 0, 1
BLOCK = 128                      # columns that share a scale in an 8-bit checkpoint
MAX_GROUPS = 1024
_TYPES = {torch.bfloat16: BF16, torch.float32: F32}


def _round_up(n: int, m: int) -> int:
    return -(-n // m) * m


class PackedActivations:
    """M x k activations in 8 bits: q (int8, rows 16-byte aligned) counts units of 2 ** (scales - 127), one unit for each
    128 columns of a row; scales is ceil(k / 128) x M.  A value that was not finite has q = -128, its block the scale 255, and the
    block reads as NaN."""

    __slots__ = ("shape", "_buffer", "_q", "_scales", "_at", "_ld", "_scales_at")

    @classmethod
    def _of(cls, buffer, M, k):
        """One buffer: the whole numbers' rows, then the scales."""
        self = cls.__new__(cls)
        self.shape, self._buffer, self._ld = (M, k), buffer, _round_up(k, 16)
        self._at = buffer.data_ptr()
        self._scales_at = self._at + M * self._ld
        self._q = self._scales = None
        return self

    @classmethod
    def from_parts(cls, q, scales):
        """A checkpoint made elsewhere (a restored file, another process).  No copy."""
        M, k = q.shape
        if q.dtype != torch.int8 or scales.dtype != torch.uint8 or tuple(scales.shape) != (-(-k // BLOCK), M):
            raise ValueError("q: M x k int8 and scales: ceil(k / 128) x M uint8 are needed")
        if not scales.is_contiguous() or (q.numel() and (q.stride(1) != 1 or (M > 1 and (q.stride(0) % 16 or q.stride(0) < k)) or q.data_ptr() % 16)) \
                or q.device != scales.device:
            raise ValueError("q needs 16-byte aligned rows, scales has to be contiguous and on the same device")
        self = cls.__new__(cls)
        self.shape, self._ld = (M, k), q.stride(0) if M > 1 else _round_up(k, 16)
        self._buffer, self._q, self._scales = q, q, scales
        self._at, self._scales_at = q.data_ptr(), scales.data_ptr()
        return self

    def __reduce__(self):
        """Copies and pickles hold tensors of their own, and the addresses of those."""
        return PackedActivations.from_parts, (self.q, self.scales)

    @property
    def q(self):
        if self._q is None:
            M, k = self.shape
            self._q = self._buffer[:M * self._ld].view(torch.int8).view(M, self._ld)[:, :k]
        return self._q

    @property
    def scales(self):
        if self._scales is None:
            M, k = self.shape
            self._scales = self._buffer[M * self._ld:].view(-(-k // BLOCK), M)
        return self._scales


class LMOps:
    """The operators, with the scratch their kernels share: order the calls of one object (one stream, or events)."""

    def __init__(self, workspace_limit: int = 2 << 30, widen: bool = True):
        """workspace_limit: bytes that a call of the vocabulary operators may take for what it keeps of the rows it works on
        at a time (a longer batch is worked on in several passes).  widen: a weight gradient from a large checkpoint may take
        room for the checkpoint in bf16, with which it is faster."""
        self.workspace_limit, self.widen = int(workspace_limit), bool(widen)
        if not torch.cuda.is_available():
            raise RuntimeError("the language-model operators need a CUDA device (there is no CPU fallback)")
        self._lib = _E.load()
        from . import _lm_binding
        self._b = _lm_binding
        h = ctypes.c_void_p()
        rc = self._lib.cocod_lm_create(ctypes.byref(h))
        if rc != _E.OK:
            raise _E.CocodError(rc, "cocod_lm_create")
        self._h = h.value
        self._device = torch.cuda.current_device()

    @staticmethod
    def _checked(result, name):
        if type(result) is int:
            raise _E.CocodError(result, name)
        return result

    @staticmethod
    def _code(out_dtype):
        if out_dtype is None:
            return -1
        if out_dtype not in _TYPES:
            raise ValueError(f"result type {out_dtype}: bfloat16 or float32")
        return _TYPES[out_dtype]

    # ------------------------------------------------------------------------------------------ products by group
    # All calls run on torch's current stream.
    def grouped_forward(self, x, w, offsets, out=None, out_dtype=None):
        """y[m] = w[g] x[m] for the rows m of every group g.  x: M x k bf16, w: G x n x k bf16 (any group and row stride),
        offsets: G + 1 int32; y: bf16 unless out_dtype or out says float32.  Rows behind offsets[G] are not written."""
        y = self._b.grouped_forward(self._h, self._device, x, w, offsets, out, -1 if out_dtype is None else self._code(out_dtype))
        return y if type(y) is not int else self._checked(y, "cocod_grouped_forward")

    def grouped_input_grad(self, dy, w, offsets, out=None, out_dtype=None):
        """dx[m] = w[g]^T dy[m]: the gradient of grouped_forward's input.  dy: M x n bf16."""
        dx = self._b.grouped_input_grad(self._h, self._device, dy, w, offsets, out, -1 if out_dtype is None else self._code(out_dtype))
        return dx if type(dx) is not int else self._checked(dx, "cocod_grouped_input_grad")

    def grouped_weight_grad(self, dy, x, offsets, out=None, out_dtype=None):
        """dw[g] = sum over the group's rows of dy[m] x[m]^T: the gradient of grouped_forward's weights, G x n x k, 0 for an
        empty group; float32 unless out_dtype or out says bf16.  x: M x k bf16, or the PackedActivations kept of it.  out: any
        group and row stride, e.g. a view of the K x P gradients that Engine.local_step takes."""
        code = -1 if out_dtype is None else self._code(out_dtype)
        if isinstance(x, PackedActivations):
            self._here(x)
            dw = self._b.grouped_weight_grad_packed(self._h, self._device, dy, x.shape[0], x.shape[1], x._at, x._ld, x._scales_at, offsets, out,
                                                    code, self.widen)
        else:
            dw = self._b.grouped_weight_grad(self._h, self._device, dy, x, offsets, out, code)
        return dw if type(dw) is not int else self._checked(dw, "cocod_grouped_weight_grad")

    # ------------------------------------------------------------------------------------------ activations in 8 bits
    def _here(self, packed):
        if packed._buffer.get_device() != self._device:
            raise ValueError(f"checkpoint: on {packed._buffer.device}, need cuda:{self._device} (the current device at creation)")

    def act_pack(self, x, out=None):
        """The 8-bit form of x (M x k bf16)."""
        if out is None:
            buffer = self._checked(self._b.act_pack_new(self._h, self._device, x), "cocod_act_pack")
            return PackedActivations._of(buffer, *x.shape)
        self._here(out)
        rc = self._b.act_pack_into(self._h, self._device, x, out.shape[0], out.shape[1], out._at, out._ld, out._scales_at)
        if rc != _E.OK:
            raise _E.CocodError(rc, "cocod_act_pack")
        return out

    def act_unpack(self, packed, out=None):
        """The bf16 values that a checkpoint stands for."""
        self._here(packed)
        return self._checked(self._b.act_unpack(self._h, self._device, packed._buffer, packed.shape[0], packed.shape[1], packed._at, packed._ld,
                                                packed._scales_at, out), "cocod_act_unpack")

    def act_relu_grad(self, dh, packed, out=None):
        """dz = dh where the kept activation is positive, 0 elsewhere (NaN where it was not finite).  out may be dh."""
        self._here(packed)
        return self._checked(self._b.act_relu_grad(self._h, self._device, dh, packed.shape[0], packed.shape[1], packed._at, packed._ld, out),
                             "cocod_act_relu_grad")

    # ------------------------------------------------------------------------------------------ vocabulary
    def vocab_loss(self, x, w, labels, offsets, row_weights=None):
        """(loss of each group, loss of each row) of softmax cross-entropy with logits x w[g]^T.  x: M x D bf16, w: G x V x D bf16,
        labels: M int32, negative for rows that take no part; the mean over a group's other rows, or the sum weighted by
        row_weights (M float32)."""
        return self._checked(self._b.vocab_loss(self._h, self._device, x, w, labels, offsets, row_weights, self.workspace_limit), "cocod_vocab_loss")

    def vocab_loss_grad(self, x, w, labels, offsets, row_weights=None, dw=None, dw_dtype=None):
        """(loss, row_loss, dx, dw): vocab_loss and the gradients of the groups' losses.  dw: G x V x D, bf16 (as w) or float32, for
        example a view of the K x P gradients that Engine.local_step takes."""
        return self._checked(self._b.vocab_loss_grad(self._h, self._device, x, w, labels, offsets, row_weights, self.workspace_limit, dw,
                                                     self._code(dw_dtype)), "cocod_vocab_loss_grad")

    # ------------------------------------------------------------------------------------------ the rest
    def check(self):
        """Synchronise the current stream; raise if a kernel gave up a wait or met offsets or labels out of range."""
        rc = self._lib.cocod_lm_check(self._h, torch.cuda.current_stream(self._device).cuda_stream)
        if rc != _E.OK:
            raise _E.CocodError(rc, "cocod_lm_check")

    @property
    def launch_count(self) -> int:
        return int(self._lib.cocod_lm_launch_count(self._h))

    def destroy(self):
        if getattr(self, "_h", 0):
            h, self._h = self._h, 0
            self._lib.cocod_lm_destroy(h)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def grouped_wait_selftest(wait_ms: int = 50, pair: bool = True) -> int:
    """Run the bounded-wait self-test of the product kernels; returns the library's code (ERR_TIMEOUT is the expected one)."""
    return int(_E.load().cocod_grouped_wait_selftest(int(wait_ms), int(pair), torch.cuda.current_stream().cuda_stream))
