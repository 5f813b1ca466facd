"""Python binding of the operators declared in ``include/zo_ops.h``.

Argument marshalling only, with the C names: matrices in microscaled 4-bit
floating point (``Mx4``) and their products, a teacher's top logits, the
distillation loss with the gradient of the student's logits.  Device buffers
are torch tensors; two-dimensional ones may have any row stride as long as
their rows are contiguous.  Every call checks element types, shapes and
devices before anything reaches the device and enqueues on ``stream`` (torch's
current stream by default).  On another stream than the current one the
tensors are recorded as in use there; ordering the streams stays with the
caller.
"""
import ctypes

import torch

from . import ZoError, ZO_EHIP, ZO_OK, _Distill, _Mx4, lib

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _size(n, where):
    if n < 0:
        raise ZoError(int(n), where)
    return int(n)


def zo_mx4_code_bytes(rows, cols):
    """Bytes of the codes of a rows x cols 4-bit matrix."""
    return _size(lib().zo_mx4_code_bytes(int(rows), int(cols)), "zo_mx4_code_bytes")


def zo_mx4_scale_bytes(rows, cols):
    """Bytes of the scales of a rows x cols 4-bit matrix."""
    return _size(lib().zo_mx4_scale_bytes(int(rows), int(cols)), "zo_mx4_scale_bytes")


def zo_top_logits_ws(rows, vocab, top):
    """Bytes of workspace of zo_top_logits."""
    return _size(lib().zo_top_logits_ws(int(rows), int(vocab), int(top)), "zo_top_logits_ws")


def zo_distill_ws(rows, vocab):
    """Bytes of workspace of zo_distill_loss."""
    return _size(lib().zo_distill_ws(int(rows), int(vocab)), "zo_distill_ws")


class Mx4:
    """A rows x cols matrix in microscaled 4-bit floating point: ``codes`` and
    ``scales``, uint8 device tensors in the layout of ``zo_mx4`` (allocated when
    not given).  Its rows are the axis that products reduce over."""

    __slots__ = ("rows", "cols", "codes", "scales", "_c")

    def __init__(self, rows, cols, codes=None, scales=None, device="cuda"):
        self.rows, self.cols = int(rows), int(cols)
        nc, ns = zo_mx4_code_bytes(rows, cols), zo_mx4_scale_bytes(rows, cols)
        if codes is None:
            codes = torch.empty(nc, dtype=torch.uint8, device=device)
        if scales is None:
            scales = torch.empty(ns, dtype=torch.uint8, device=codes.device)
        for t, n, what in ((codes, nc, "codes"), (scales, ns, "scales")):
            if t.dtype != torch.uint8:
                raise ValueError(f"{what}: expected uint8, got {t.dtype}")
            if not t.is_contiguous() or t.numel() < n:
                raise ValueError(f"{what}: needs {n} contiguous elements, has {t.numel()}")
        self.codes, self.scales = codes, scales
        self._c = _Mx4(codes.data_ptr(), scales.data_ptr(), self.rows, self.cols)


class _Call:
    """One call's tensors: all on one device, recorded on the call's stream."""

    def __init__(self, where, stream):
        self.where, self.stream, self.tensors = where, stream, []

    def add(self, t, what):
        if not t.is_cuda:
            raise ValueError(f"{what}: expected a device tensor")
        if self.tensors and t.device != self.tensors[0].device:
            raise ValueError(f"{what}: on {t.device}, expected {self.tensors[0].device}")
        self.tensors.append(t)
        return t.data_ptr()

    def mx4(self, q, what):
        if not isinstance(q, Mx4):
            raise ValueError(f"{what}: expected an Mx4")
        self.add(q.codes, what)
        self.add(q.scales, what)
        return ctypes.addressof(q._c)

    def matrix(self, t, what, rows=None, cols=None):
        """(pointer, type, rows, cols, row stride)"""
        code = _DTYPES.get(t.dtype)
        if code is None:
            raise ValueError(f"{what}: expected float32, float16 or bfloat16, got {t.dtype}")
        if t.dim() != 2 or (rows is not None and tuple(t.shape) != (rows, cols)):
            raise ValueError(f"{what}: expected shape {(rows, cols) if rows is not None else '2-d'}"
                             f", got {tuple(t.shape)}")
        r, c = t.shape
        ld = t.stride(0) if r > 1 else max(c, 1)
        if c > 1 and t.stride(1) != 1:
            raise ValueError(f"{what}: expected contiguous rows")
        if r > 1 and ld < c:
            raise ValueError(f"{what}: rows overlap")
        return self.add(t, what), code, r, c, max(ld, 1)

    def vector(self, t, what, dtype, shape):
        if t is None:
            return None
        if t.dtype != dtype:
            raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
        if tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError(f"{what}: expected contiguous {shape}, got {tuple(t.shape)}")
        return self.add(t, what)

    def workspace(self, ws, nbytes):
        """The caller's workspace, or one from torch's allocator on the call's stream."""
        if nbytes == 0:
            return None, 0
        if ws is None:
            dev = self.tensors[0].device
            with torch.cuda.stream(self.stream):
                ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        elif ws.dtype != torch.uint8 or not ws.is_contiguous() or ws.numel() < nbytes:
            raise ValueError(f"ws: needs {nbytes} contiguous uint8 elements")
        return self.add(ws, "ws"), ws.numel()

    def run(self, *args):
        dev = self.tensors[0].device
        if dev.index == torch.cuda.current_device():
            rc = self._launch(args)
        else:
            with torch.cuda.device(dev):
                rc = self._launch(args)
        if rc != ZO_OK:
            detail = lib().zo_ops_last_hip_error().decode() if rc == ZO_EHIP else ""
            raise ZoError(rc, self.where, detail)

    def _launch(self, args):
        current = torch.cuda.current_stream()
        s = current if self.stream is None else self.stream
        rc = getattr(lib(), self.where)(*args, s.cuda_stream)
        if self.stream is not None and s != current:
            for t in self.tensors:
                t.record_stream(s)
        return rc


def zo_mx4_quantize(x, q=None, qt=None, stream=None):
    """x [rows, cols] into q (an Mx4 of rows x cols, blocks along x's rows) and / or
    qt (cols x rows, blocks along x's columns), reading x once."""
    c = _Call("zo_mx4_quantize", stream)
    p, dt, rows, cols, ld = c.matrix(x, "x")
    c.run(p, dt, rows, cols, ld, c.mx4(q, "q") if q is not None else None,
          c.mx4(qt, "qt") if qt is not None else None)


def zo_mx4_dequantize(q, out, stream=None):
    """The values of q into out [q.rows, q.cols]."""
    c = _Call("zo_mx4_dequantize", stream)
    pq = c.mx4(q, "q")
    p, dt, _, _, ld = c.matrix(out, "out", q.rows, q.cols)
    c.run(pq, p, dt, ld)


def zo_mx4_product(a, b, out, stream=None):
    """out [a.rows, b.rows] = a b^T, reduced over the columns of both."""
    c = _Call("zo_mx4_product", stream)
    pa, pb = c.mx4(a, "a"), c.mx4(b, "b")
    p, dt, _, _, ld = c.matrix(out, "out", a.rows, b.rows)
    c.run(pa, pb, p, dt, ld)


def zo_mx4_linear(x, w, out, xq, stream=None):
    """out [rows, w.rows] = x quantised along its rows times w^T; xq (an Mx4 of
    x's shape) is workspace."""
    c = _Call("zo_mx4_linear", stream)
    pw, pq = c.mx4(w, "w"), c.mx4(xq, "xq")
    px, dx, rows, _, ldx = c.matrix(x, "x", xq.rows, xq.cols)
    po, do, _, _, ldo = c.matrix(out, "out", rows, w.rows)
    c.run(px, dx, ldx, pw, pq, po, do, ldo)


def zo_top_logits(z, values, columns, lse=None, *, tau=1.0, ws=None, stream=None):
    """The values.shape[1] largest logits of every row of z [rows, vocab] in
    descending order (ties: lowest column first) into values (float32), their
    columns into columns (int32), and log sum exp(z / tau) into lse [rows]."""
    c = _Call("zo_top_logits", stream)
    p, dt, rows, vocab, ld = c.matrix(z, "z")
    if values.dim() != 2:
        raise ValueError("values: expected a matrix")
    shape = (rows, int(values.shape[1]))
    pv = c.vector(values, "values", torch.float32, shape)
    pc = c.vector(columns, "columns", torch.int32, shape)
    pl = c.vector(lse, "lse", torch.float32, (rows,))
    pw, nw = c.workspace(ws, zo_top_logits_ws(rows, vocab, shape[1]))
    c.run(p, dt, rows, vocab, ld, shape[1], float(tau), pv, pc, pl, pw, nw)


def zo_distill_loss(z, values, columns, loss=None, dz=None, *, tau=1.0, teacher_lse=None,
                    labels=None, kd_weight=1.0, ce_weight=0.0, row_weight=None, ws=None,
                    stream=None):
    """Distillation from a teacher's top logits: the loss of every row of the
    student's logits z [rows, vocab] into loss (float32 [rows]) and / or its
    gradient into dz (z's type and shape; may be z itself).

    values (float32) and columns (int32), [rows, top], are the teacher's; a
    column outside the vocabulary marks an unused slot.  teacher_lse adds the
    rest of the teacher's mass as one outcome.  labels (int32 [rows], outside
    the vocabulary: none) enter with ce_weight; row_weight (float32 [rows]) is
    the gradient from above, rows of weight 0 are skipped."""
    c = _Call("zo_distill_loss", stream)
    p, dt, rows, vocab, ldz = c.matrix(z, "z")
    if values.dim() != 2:
        raise ValueError("values: expected a matrix")
    shape = (rows, int(values.shape[1]))
    a = _Distill(z=p, dtype=dt, rows=rows, vocab=vocab, ldz=ldz, top=shape[1],
                 values=c.vector(values, "values", torch.float32, shape),
                 columns=c.vector(columns, "columns", torch.int32, shape),
                 teacher_lse=c.vector(teacher_lse, "teacher_lse", torch.float32, (rows,)),
                 labels=c.vector(labels, "labels", torch.int32, (rows,)),
                 row_weight=c.vector(row_weight, "row_weight", torch.float32, (rows,)),
                 tau=float(tau), kd_weight=float(kd_weight), ce_weight=float(ce_weight),
                 loss=c.vector(loss, "loss", torch.float32, (rows,)))
    if dz is not None:
        if dz.dtype != z.dtype:
            raise ValueError(f"dz: expected {z.dtype}, got {dz.dtype}")
        a.dz, _, _, _, a.lddz = c.matrix(dz, "dz", rows, vocab)
    a.ws, a.ws_bytes = c.workspace(ws, zo_distill_ws(rows, vocab))
    c.run(ctypes.byref(a))
