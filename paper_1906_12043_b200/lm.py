"""Thin ctypes binding over the language-model operators of libcocod.so (include/cocod_lm.h).

Marshalling only: every product, sum and exponential is computed by the library's CUDA kernels.  torch is used for
device memory and streams.  No CPU fallback.

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
_SIZES = {torch.bfloat16: 2, torch.float32: 4}
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _round_up(n: int, m: int) -> int:
    return -(-n // m) * m


class PackedActivations:
    """M x k activations in 8 bits: q (int8, rows 16-byte aligned) counts units of 2 ** (scales - 127), one unit for each
    128 columns of a row; scales is ceil(k / 128) x M.  A value that was not finite has q = -128, its block the scale 255, and the
    block reads as NaN."""

    __slots__ = ("shape", "_buffer", "_q", "_scales", "_at", "_ld", "_scales_at")

    def __init__(self, M: int, k: int, like):
        """Room for M x k values on the device of `like`: one buffer, the whole numbers' rows first."""
        ld = _round_up(k, 16)
        self.shape, self._ld = (M, k), ld
        self._buffer = like.new_empty(M * ld + -(-k // BLOCK) * M, dtype=torch.uint8)
        self._at = self._buffer.data_ptr()
        self._scales_at = self._at + M * ld
        self._q = self._scales = None

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
        h = ctypes.c_void_p()
        rc = self._lib.cocod_lm_create(ctypes.byref(h))
        if rc != _E.OK:
            raise _E.CocodError(rc, "cocod_lm_create")
        self._h = h
        self._device = torch.cuda.current_device()

    # ------------------------------------------------------------------------------------------ arguments
    def _rows(self, t, name, M, cols, dtype=torch.bfloat16, align=16):
        """(address, row stride) of an M x cols matrix with contiguous rows that start at multiples of `align` bytes."""
        if t.dtype is dtype and t.get_device() == self._device and t.shape == (M, cols):
            ld, step = t.stride()
            if M <= 1:
                ld = _round_up(cols, 16)
            at = t.data_ptr()
            if (step == 1 or cols == 1) and ld >= cols and not (at | ld * _SIZES[dtype]) % align:
                return at, ld
        raise ValueError(f"{name}: need {M} x {cols} {dtype} on cuda:{self._device} (the current device at creation), rows contiguous, not "
                         f"overlapping and starting at multiples of {align} bytes; got {tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}")

    def _groups(self, t, name, G, n, k, dtype=torch.bfloat16):
        """(address, row stride, group stride) of one n x k matrix per group."""
        if t.dtype is dtype and t.get_device() == self._device and t.shape == (G, n, k):
            gs, ld, step = t.stride()
            if n == 1:
                ld = _round_up(k, 8)
            if G == 1:
                gs = n * ld
            at, size = t.data_ptr(), _SIZES[dtype]
            if (step == 1 or k == 1) and ld >= k and gs >= (n - 1) * ld + k and not (at | ld * size | gs * size) % 16:
                return at, ld, gs
        raise ValueError(f"{name}: need {G} x {n} x {k} {dtype} on cuda:{self._device} (the current device at creation), rows contiguous, rows and "
                         f"groups not overlapping and starting at multiples of 16 bytes; got {tuple(t.shape)} {t.dtype} on {t.device}, strides {t.stride()}")

    def _vector(self, t, name, n, dtype):
        if t.dtype is dtype and t.get_device() == self._device and t.shape == (n,) and (n <= 1 or t.stride() == (1,)):
            return t.data_ptr()
        raise ValueError(f"{name}: need {n} contiguous {dtype} on cuda:{self._device} (the current device at creation); got {tuple(t.shape)} "
                         f"{t.dtype} on {t.device}")

    @staticmethod
    def _type(out, out_dtype, usual):
        dtype = out_dtype or (usual if out is None else out.dtype)
        if dtype not in _TYPES or (out is not None and out.dtype is not dtype):
            raise ValueError(f"result type {dtype}{'' if out is None else f' for a result of {out.dtype}'}: bfloat16 or float32, as the result")
        return dtype

    def _call(self, name, function, *args):
        rc = function(self._h, *args, _raw_stream(self._device))
        if rc != _E.OK:
            raise _E.CocodError(rc, name)

    # ------------------------------------------------------------------------------------------ products by group
    # All calls run on torch's current stream.
    def grouped_forward(self, x, w, offsets, out=None, out_dtype=None):
        """y[m] = w[g] x[m] for the rows m of every group g.  x: M x k bf16, w: G x n x k bf16 (any group and row stride),
        offsets: G + 1 int32.  Rows behind offsets[G] are not written."""
        G, n, k = w.shape
        M = x.shape[0]
        out, dtype, at, ld = self._result(x, M, n, out, out_dtype)
        self._call("cocod_grouped_forward", self._lib.cocod_grouped_forward, G, self._vector(offsets, "offsets", G + 1, torch.int32), M, n, k,
                   *self._rows(x, "x", M, k), *self._groups(w, "w", G, n, k), at, ld, _TYPES[dtype])
        return out

    def grouped_input_grad(self, dy, w, offsets, out=None, out_dtype=None):
        """dx[m] = w[g]^T dy[m]: the gradient of grouped_forward's input.  dy: M x n bf16."""
        G, n, k = w.shape
        M = dy.shape[0]
        out, dtype, at, ld = self._result(dy, M, k, out, out_dtype)
        self._call("cocod_grouped_input_grad", self._lib.cocod_grouped_input_grad, G, self._vector(offsets, "offsets", G + 1, torch.int32), M, n, k,
                   *self._rows(dy, "dy", M, n), *self._groups(w, "w", G, n, k), at, ld, _TYPES[dtype])
        return out

    def _result(self, like, M, cols, out, out_dtype):
        """(result, its type, address, row stride): a new M x cols matrix, or the caller's after a look."""
        if out is None:
            dtype = self._type(None, out_dtype, torch.bfloat16)
            out = like.new_empty((M, cols), dtype=dtype)
            return out, dtype, out.data_ptr(), cols
        dtype = self._type(out, out_dtype, None)
        return (out, dtype, *self._rows(out, "out", M, cols, dtype))

    def grouped_weight_grad(self, dy, x, offsets, out=None, out_dtype=None):
        """dw[g] = sum over the group's rows of dy[m] x[m]^T: the gradient of grouped_forward's weights, G x n x k, 0 for an
        empty group.  x: M x k bf16, or the PackedActivations kept of it.  out: any group and row stride, e.g. a view of the
        K x P gradients that Engine.local_step takes."""
        M, k = x.shape
        n, G = dy.shape[1], offsets.shape[0] - 1
        dtype = self._type(out, out_dtype, torch.float32)
        if out is None:
            out = dy.new_empty((G, n, k), dtype=dtype)
            result = out.data_ptr(), k, n * k
        else:
            result = self._groups(out, "out", G, n, k, dtype)
        shape = (G, self._vector(offsets, "offsets", G + 1, torch.int32), M, n, k, *self._rows(dy, "dy", M, n))
        if isinstance(x, PackedActivations):
            ws = self._scratch(self._lib.cocod_grouped_packed_workspace(G, M, n, k)) if self.widen else None
            self._call("cocod_grouped_weight_grad_packed", self._lib.cocod_grouped_weight_grad_packed, *shape,
                       *self._kept(x, M, k), x._scales_at, *result, _TYPES[dtype],
                       None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel())
        else:
            self._call("cocod_grouped_weight_grad", self._lib.cocod_grouped_weight_grad, *shape, *self._rows(x, "x", M, k), *result, _TYPES[dtype])
        return out

    def _scratch(self, nbytes):
        if nbytes < 0:
            raise ValueError("sizes outside the operators' range")
        return torch.empty(nbytes, dtype=torch.uint8, device=self._device) if nbytes else None

    # ------------------------------------------------------------------------------------------ activations in 8 bits
    def act_pack(self, x, out=None):
        """The 8-bit form of x (M x k bf16)."""
        M, k = x.shape
        if out is None:
            out = PackedActivations(M, k, x)
        self._call("cocod_act_pack", self._lib.cocod_act_pack, M, k, *self._rows(x, "x", M, k, align=1), *self._kept(out, M, k), out._scales_at)
        return out

    def _kept(self, packed, M, k):
        """(address, row stride) of a checkpoint's whole numbers."""
        if packed.shape == (M, k) and packed._buffer.get_device() == self._device:
            return packed._at, packed._ld
        raise ValueError(f"checkpoint: need {M} x {k} on cuda:{self._device}, got {packed.shape} on {packed._buffer.device}")

    def act_unpack(self, packed, out=None):
        """The bf16 values that a checkpoint stands for."""
        M, k = packed.shape
        if out is None:
            out = packed._buffer.new_empty((M, k), dtype=torch.bfloat16)
            at, ld = out.data_ptr(), k
        else:
            at, ld = self._rows(out, "out", M, k, align=1)
        self._call("cocod_act_unpack", self._lib.cocod_act_unpack, M, k, *self._kept(packed, M, k), packed._scales_at, at, ld)
        return out

    def act_relu_grad(self, dh, packed, out=None):
        """dz = dh where the kept activation is positive, 0 elsewhere (NaN where it was not finite).  out may be dh."""
        M, k = packed.shape
        given = self._rows(dh, "dh", M, k, align=1)
        if out is None:
            out = dh.new_empty((M, k))
            at, ld = out.data_ptr(), k
        else:
            at, ld = self._rows(out, "out", M, k, align=1)
        self._call("cocod_act_relu_grad", self._lib.cocod_act_relu_grad, M, k, *given, *self._kept(packed, M, k), at, ld)
        return out

    # ------------------------------------------------------------------------------------------ vocabulary
    def _vocab(self, x, w, labels, offsets, row_weights):
        G, V, D = w.shape
        M = x.shape[0]
        loss, row_loss = x.new_empty(G, dtype=torch.float32), x.new_empty(M, dtype=torch.float32)
        return loss, row_loss, (G, self._vector(offsets, "offsets", G + 1, torch.int32), M, V, D, *self._rows(x, "x", M, D),
                                *self._groups(w, "w", G, V, D), self._vector(labels, "labels", M, torch.int32),
                                None if row_weights is None else self._vector(row_weights, "row_weights", M, torch.float32),
                                loss.data_ptr(), row_loss.data_ptr())

    def vocab_loss(self, x, w, labels, offsets, row_weights=None):
        """(loss of each group, loss of each row) of softmax cross-entropy with logits x w[g]^T.  x: M x D bf16, w: G x V x D bf16,
        labels: M int32, negative for rows that take no part; the mean over a group's other rows, or the sum weighted by
        row_weights (M float32)."""
        loss, row_loss, args = self._vocab(x, w, labels, offsets, row_weights)
        G, _, M, V, D = args[:5]
        ws = self._scratch(self._lib.cocod_vocab_workspace(G, M, V, D, 0, BF16, self.workspace_limit))
        self._call("cocod_vocab_loss", self._lib.cocod_vocab_loss, *args, ws.data_ptr(), ws.numel())
        return loss, row_loss

    def vocab_loss_grad(self, x, w, labels, offsets, row_weights=None, dw=None, dw_dtype=None):
        """(loss, row_loss, dx, dw): vocab_loss and the gradients of the groups' losses.  dw: G x V x D, bf16 (as w) or float32, for
        example a view of the K x P gradients that Engine.local_step takes."""
        dtype = self._type(dw, dw_dtype, torch.bfloat16)
        loss, row_loss, args = self._vocab(x, w, labels, offsets, row_weights)
        G, _, M, V, D = args[:5]
        dx = x.new_empty((M, D))
        if dw is None:
            dw = x.new_empty((G, V, D), dtype=dtype)
            result = dw.data_ptr(), D, V * D
        else:
            result = self._groups(dw, "dw", G, V, D, dtype)
        ws = self._scratch(self._lib.cocod_vocab_workspace(G, M, V, D, 1, _TYPES[dtype], self.workspace_limit))
        self._call("cocod_vocab_loss_grad", self._lib.cocod_vocab_loss_grad, *args, dx.data_ptr(), D,
                   *result, _TYPES[dtype], ws.data_ptr(), ws.numel())
        return loss, row_loss, dx, dw

    # ------------------------------------------------------------------------------------------ the rest
    def check(self):
        """Synchronise the current stream; raise if a kernel gave up a wait or met offsets or labels out of range."""
        rc = self._lib.cocod_lm_check(self._h, _raw_stream(self._device))
        if rc != _E.OK:
            raise _E.CocodError(rc, "cocod_lm_check")

    @property
    def launch_count(self) -> int:
        return int(self._lib.cocod_lm_launch_count(self._h))

    def destroy(self):
        if getattr(self, "_h", None):
            h, self._h = self._h, None
            self._lib.cocod_lm_destroy(h)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def grouped_wait_selftest(wait_ms: int = 50, pair: bool = True) -> int:
    """Run the bounded-wait self-test of the product kernels; returns the library's code (ERR_TIMEOUT is the expected one)."""
    return int(_E.load().cocod_grouped_wait_selftest(int(wait_ms), int(pair), torch.cuda.current_stream().cuda_stream))
