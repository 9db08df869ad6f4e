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
FORWARD, INPUT_GRAD, WEIGHT_GRAD = 0, 1, 2
BLOCK = 128                      # columns that share a scale in an 8-bit checkpoint
MAX_GROUPS = 1024
_TYPES = {torch.bfloat16: BF16, torch.float32: F32}


def _round_up(n: int, m: int) -> int:
    return -(-n // m) * m


class PackedActivations:
    """M x k activations in 8 bits: q (int8, rows 16-byte aligned) counts units of 2 ** (scales - 127), one unit for each
    128 columns of a row; scales is ceil(k / 128) x M.  A value that was not finite has q = -128 and reads as NaN."""

    __slots__ = ("q", "scales", "shape")

    def __init__(self, M: int, k: int, device):
        self.q = torch.empty((M, _round_up(k, 16)), dtype=torch.int8, device=device)[:, :k]
        self.scales = torch.empty((-(-k // BLOCK), M), dtype=torch.uint8, device=device)
        self.shape = (M, k)

    @classmethod
    def from_parts(cls, q, scales):
        """A checkpoint made elsewhere (a restored file, another process).  No copy."""
        M, k = q.shape
        if q.dtype != torch.int8 or scales.dtype != torch.uint8 or tuple(scales.shape) != (-(-k // BLOCK), M):
            raise ValueError("q: M x k int8 and scales: ceil(k / 128) x M uint8 are needed")
        if not scales.is_contiguous() or (q.numel() and (q.stride(1) != 1 or (M > 1 and q.stride(0) % 16) or q.data_ptr() % 16)):
            raise ValueError("q needs 16-byte aligned rows, scales has to be contiguous")
        self = cls.__new__(cls)
        self.q, self.scales, self.shape = q, scales, (M, k)
        return self


class LMOps:
    """The operators, with the scratch their kernels share: order the calls of one object (one stream, or events)."""

    def __init__(self, workspace_limit: int = 2 << 30):
        """workspace_limit: bytes that a call of the vocabulary operators may take for what it keeps of the rows it works on
        at a time (a longer batch is worked on in several passes)."""
        self.workspace_limit = int(workspace_limit)
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
    def _rows(self, t, name, M=None, cols=None, dtype=torch.bfloat16, align=16):
        """(address, row stride) of a matrix with contiguous rows."""
        if t.dim() != 2 or t.dtype is not dtype or t.device.type != "cuda" or t.device.index != self._device:
            raise ValueError(f"{name}: need a two-dimensional {dtype} tensor on cuda:{self._device}, the current device at creation")
        if (M is not None and t.shape[0] != M) or (cols is not None and t.shape[1] != cols):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, need {M if M is not None else 'any'} x {cols if cols is not None else 'any'}")
        if t.shape[1] > 1 and t.stride(1) != 1:
            raise ValueError(f"{name}: rows have to be contiguous")
        ld = t.stride(0) if t.shape[0] > 1 else _round_up(t.shape[1], 16)
        if align and (t.data_ptr() % align or ld * t.element_size() % align):
            raise ValueError(f"{name}: rows have to start at multiples of {align} bytes")
        if ld < t.shape[1]:
            raise ValueError(f"{name}: rows overlap")
        return t.data_ptr(), ld

    def _groups(self, t, name, shape=None, dtype=torch.bfloat16):
        """(address, row stride, group stride) of one matrix per group."""
        if t.dim() != 3 or t.dtype is not dtype or t.device.type != "cuda" or t.device.index != self._device:
            raise ValueError(f"{name}: need a three-dimensional {dtype} tensor on cuda:{self._device}, the current device at creation")
        if shape is not None and tuple(t.shape) != tuple(shape):
            raise ValueError(f"{name}: shape {tuple(t.shape)}, need {tuple(shape)}")
        G, n, k = t.shape
        if k > 1 and t.stride(2) != 1:
            raise ValueError(f"{name}: rows have to be contiguous")
        ld = t.stride(1) if n > 1 else _round_up(k, 8)
        gs = t.stride(0) if G > 1 else n * ld
        if t.data_ptr() % 16 or ld * t.element_size() % 16 or gs * t.element_size() % 16:
            raise ValueError(f"{name}: rows and groups have to start at multiples of 16 bytes")
        if ld < k or gs < (n - 1) * ld + k:
            raise ValueError(f"{name}: rows or groups overlap")
        return t.data_ptr(), ld, gs

    def _offsets(self, offsets, G):
        if offsets.dim() != 1 or offsets.dtype is not torch.int32 or offsets.shape[0] != G + 1 or not offsets.is_contiguous() \
                or offsets.device.type != "cuda" or offsets.device.index != self._device:
            raise ValueError(f"offsets: need {G + 1} contiguous int32 on cuda:{self._device} (one more than there are groups)")
        return offsets.data_ptr()

    def _type(self, out, out_dtype):
        dtype = out.dtype if out is not None else out_dtype
        if dtype not in _TYPES or (out is not None and out_dtype not in (None, dtype)):
            raise ValueError(f"result type {out_dtype if out is None else (out.dtype, out_dtype)}: bfloat16 or float32")
        return dtype

    def _scratch(self, nbytes):
        if nbytes < 0:
            raise ValueError("sizes outside the operators' range")
        return torch.empty(nbytes, dtype=torch.uint8, device=self._device) if nbytes else None

    @staticmethod
    def _addr(t):
        return None if t is None else t.data_ptr()

    def _call(self, name, *args):
        rc = getattr(self._lib, name)(self._h, *args, torch.cuda.current_stream(self._device).cuda_stream)
        if rc != _E.OK:
            raise _E.CocodError(rc, name)

    # ------------------------------------------------------------------------------------------ products by group
    # All calls run on torch's current stream.
    def grouped_forward(self, x, w, offsets, out=None, out_dtype=None):
        """y[m] = w[g] x[m] for the rows m of every group g.  x: M x k bf16, w: G x n x k bf16 (any group and row stride),
        offsets: G + 1 int32.  Rows behind offsets[G] are not written."""
        G, n, k = w.shape
        return self._rows_product("cocod_grouped_forward", FORWARD, x, "x", k, n, w, G, n, k, offsets, out, out_dtype)

    def grouped_input_grad(self, dy, w, offsets, out=None, out_dtype=None):
        """dx[m] = w[g]^T dy[m]: the gradient of grouped_forward's input.  dy: M x n bf16."""
        G, n, k = w.shape
        return self._rows_product("cocod_grouped_input_grad", INPUT_GRAD, dy, "dy", n, k, w, G, n, k, offsets, out, out_dtype)

    def _rows_product(self, name, which, a, a_name, depth, cols, w, G, n, k, offsets, out, out_dtype):
        dtype = self._type(out, out_dtype or (None if out is not None else torch.bfloat16))
        ap, lda = self._rows(a, a_name, cols=depth)
        wp, ldw, gs = self._groups(w, "w")
        M = a.shape[0]
        op = self._offsets(offsets, G)
        if out is None:
            out = torch.empty((M, cols), dtype=dtype, device=a.device)
        yp, ldy = self._rows(out, "out", M, cols, dtype)
        ws = self._scratch(self._lib.cocod_grouped_workspace(which, G, M, n, k))
        self._call(name, G, op, M, n, k, ap, lda, wp, ldw, gs, yp, ldy, _TYPES[dtype], self._addr(ws), 0 if ws is None else ws.numel())
        return out

    def grouped_weight_grad(self, dy, x, offsets, out=None, out_dtype=None):
        """dw[g] = sum over the group's rows of dy[m] x[m]^T: the gradient of grouped_forward's weights, G x n x k, 0 for an
        empty group.  x: M x k bf16, or the PackedActivations kept of it.  out: any group and row stride, e.g. a view of the
        K x P gradients that Engine.local_step takes."""
        dtype = self._type(out, out_dtype or (None if out is not None else torch.float32))
        packed = isinstance(x, PackedActivations)
        M, k = x.shape
        dp, lddy = self._rows(dy, "dy", M=M)
        n, G = dy.shape[1], offsets.shape[0] - 1
        op = self._offsets(offsets, G)
        if out is None:
            out = torch.empty((G, n, k), dtype=dtype, device=dy.device)
        wp, ldw, gs = self._groups(out, "out", (G, n, k), dtype)
        if packed:
            qp, ldq = self._rows(x.q, "x.q", M, k, torch.int8)
            ws = self._scratch(self._lib.cocod_grouped_packed_workspace(G, M, n, k))
            self._call("cocod_grouped_weight_grad_packed", G, op, M, n, k, dp, lddy, qp, ldq, x.scales.data_ptr(), wp, ldw, gs, _TYPES[dtype],
                       self._addr(ws), 0 if ws is None else ws.numel())
        else:
            xp, ldx = self._rows(x, "x")
            ws = self._scratch(self._lib.cocod_grouped_workspace(WEIGHT_GRAD, G, M, n, k))
            self._call("cocod_grouped_weight_grad", G, op, M, n, k, dp, lddy, xp, ldx, wp, ldw, gs, _TYPES[dtype], self._addr(ws),
                       0 if ws is None else ws.numel())
        return out

    # ------------------------------------------------------------------------------------------ activations in 8 bits
    def act_pack(self, x, out=None):
        """The 8-bit form of x (M x k bf16)."""
        M, k = x.shape
        xp, ldx = self._rows(x, "x", align=0)
        if out is None:
            out = PackedActivations(M, k, x.device)
        qp, ldq = self._rows(out.q, "out.q", M, k, torch.int8)
        self._call("cocod_act_pack", M, k, xp, ldx, qp, ldq, out.scales.data_ptr())
        return out

    def act_unpack(self, packed, out=None):
        """The bf16 values that a checkpoint stands for."""
        M, k = packed.shape
        if out is None:
            out = torch.empty((M, k), dtype=torch.bfloat16, device=packed.q.device)
        qp, ldq = self._rows(packed.q, "packed.q", M, k, torch.int8)
        yp, ldy = self._rows(out, "out", M, k, align=0)
        self._call("cocod_act_unpack", M, k, qp, ldq, packed.scales.data_ptr(), yp, ldy)
        return out

    def act_relu_grad(self, dh, packed, out=None):
        """dz = dh where the kept activation is positive, 0 elsewhere (NaN where it was not finite).  out may be dh."""
        M, k = packed.shape
        if out is None:
            out = torch.empty((M, k), dtype=torch.bfloat16, device=dh.device)
        dp, lddh = self._rows(dh, "dh", M, k, align=0)
        qp, ldq = self._rows(packed.q, "packed.q", M, k, torch.int8)
        zp, lddz = self._rows(out, "out", M, k, align=0)
        self._call("cocod_act_relu_grad", M, k, dp, lddh, qp, ldq, zp, lddz)
        return out

    # ------------------------------------------------------------------------------------------ vocabulary
    def _vector(self, t, name, n, dtype):
        if t.dim() != 1 or t.dtype is not dtype or t.shape[0] != n or (n > 1 and t.stride(0) != 1) or t.device.type != "cuda" \
                or t.device.index != self._device:
            raise ValueError(f"{name}: need {n} contiguous {dtype} on cuda:{self._device}")
        return t.data_ptr()

    def _vocab(self, x, w, labels, offsets, row_weights):
        G, V, D = w.shape
        M = x.shape[0]
        xp, ldx = self._rows(x, "x", cols=D)
        wp, ldw, gs = self._groups(w, "w")
        wt = None if row_weights is None else self._vector(row_weights, "row_weights", M, torch.float32)
        loss = torch.empty(G, dtype=torch.float32, device=x.device)
        row_loss = torch.empty(M, dtype=torch.float32, device=x.device)
        return loss, row_loss, (G, self._offsets(offsets, G), M, V, D, xp, ldx, wp, ldw, gs, self._vector(labels, "labels", M, torch.int32), wt,
                                loss.data_ptr(), row_loss.data_ptr())

    def vocab_loss(self, x, w, labels, offsets, row_weights=None):
        """(loss of each group, loss of each row) of softmax cross-entropy with logits x w[g]^T.  x: M x D bf16, w: G x V x D bf16,
        labels: M int32, negative for rows that take no part; the mean over a group's other rows, or the sum weighted by
        row_weights (M float32)."""
        loss, row_loss, args = self._vocab(x, w, labels, offsets, row_weights)
        G, _, M, V, D = args[:5]
        ws = self._scratch(self._lib.cocod_vocab_workspace(G, M, V, D, 0, BF16, self.workspace_limit))
        self._call("cocod_vocab_loss", *args, ws.data_ptr(), ws.numel())
        return loss, row_loss

    def vocab_loss_grad(self, x, w, labels, offsets, row_weights=None, dw=None, dw_dtype=None):
        """(loss, row_loss, dx, dw): vocab_loss and the gradients of the groups' losses.  dw: G x V x D, bf16 (as w) or float32, for
        example a view of the K x P gradients that Engine.local_step takes."""
        dtype = self._type(dw, dw_dtype or (None if dw is not None else torch.bfloat16))
        loss, row_loss, args = self._vocab(x, w, labels, offsets, row_weights)
        G, _, M, V, D = args[:5]
        dx = torch.empty((M, D), dtype=torch.bfloat16, device=x.device)
        if dw is None:
            dw = torch.empty((G, V, D), dtype=dtype, device=x.device)
        dp, lddw, gs = self._groups(dw, "dw", (G, V, D), dtype)
        ws = self._scratch(self._lib.cocod_vocab_workspace(G, M, V, D, 1, _TYPES[dtype], self.workspace_limit))
        self._call("cocod_vocab_loss_grad", *args, dx.data_ptr(), D, dp, lddw, gs, _TYPES[dtype], ws.data_ptr(), ws.numel())
        return loss, row_loss, dx, dw

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
