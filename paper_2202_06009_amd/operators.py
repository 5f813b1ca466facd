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

from . import ZoError, ZO_EHIP, ZO_EINVAL, ZO_OK, _Distill, _Mx4, lib

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_MAX_DIM = 1 << 30


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


class Mx4:
    """A rows x cols matrix in microscaled 4-bit floating point: ``codes`` and
    ``scales``, uint8 device tensors in the layout of ``zo_mx4`` (allocated when
    not given).  Its rows are the axis that products reduce over."""

    __slots__ = ("rows", "cols", "codes", "scales", "dev", "_c", "_at")

    def __init__(self, rows, cols, codes=None, scales=None, device="cuda"):
        rows, cols = int(rows), int(cols)
        if not (0 <= rows <= _MAX_DIM and 0 <= cols <= _MAX_DIM):
            raise ZoError(ZO_EINVAL, "Mx4")
        tiles = ((rows + 63) >> 6) * ((cols + 127) >> 7)     # of 64 rows x 128 columns
        if codes is None:
            codes = torch.empty(tiles * 4096, dtype=torch.uint8, device=device)
        if scales is None:
            scales = torch.empty(tiles * 256, dtype=torch.uint8, device=codes.device)
        for t, n, what in ((codes, tiles * 4096, "codes"), (scales, tiles * 256, "scales")):
            if t.dtype is not torch.uint8:
                raise ValueError(f"{what}: expected uint8, got {t.dtype}")
            if t.numel() < n or not t.is_contiguous():
                raise ValueError(f"{what}: needs {n} contiguous elements, has {t.numel()}")
        dev = codes.get_device()
        if dev < 0 or scales.get_device() != dev:
            raise ValueError("codes, scales: expected tensors on one GPU")
        self.rows, self.cols, self.codes, self.scales, self.dev = rows, cols, codes, scales, dev
        self._c = _Mx4(codes.data_ptr(), scales.data_ptr(), rows, cols)
        self._at = ctypes.addressof(self._c)


# The checks below read each attribute of a tensor once: a decode step calls
# these functions for kernels of a few microseconds.

def _at(t, what, dev):
    """Device pointer of t, which must be on device `dev`."""
    if t.get_device() != dev:
        raise ValueError(f"{what}: expected a tensor on GPU {dev}, got one on {t.device}")
    return t.data_ptr()


def _device_of(t, what):
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{what}: expected a device tensor")
    return dev


def _matrix(t, what, dev, rows=None, cols=None):
    """(pointer, element type, row stride) of a matrix with contiguous rows, of
    rows x cols when given."""
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{what}: expected float32, float16 or bfloat16, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{what}: expected a matrix, got shape {tuple(t.shape)}")
    r, c = t.shape
    if rows is not None and (r != rows or c != cols):
        raise ValueError(f"{what}: expected shape {(rows, cols)}, got {(r, c)}")
    ld, step = t.stride()
    if step != 1 and c > 1:
        raise ValueError(f"{what}: expected contiguous rows")
    if r <= 1 or c == 0:
        ld = c or 1
    elif ld < c:
        raise ValueError(f"{what}: rows overlap")
    return _at(t, what, dev), code, ld


def _vector(t, what, dev, dtype, shape):
    if t is None:
        return None
    if t.dtype is not dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what}: expected contiguous {shape}, got {tuple(t.shape)}")
    return _at(t, what, dev)


def _mx4(q, what, dev):
    """Address of q's C struct."""
    if type(q) is not Mx4:
        raise ValueError(f"{what}: expected an Mx4")
    if q.dev != dev:
        raise ValueError(f"{what}: expected an Mx4 on GPU {dev}, got one on GPU {q.dev}")
    return q._at


_functions = {}


def _run(where, dev, stream, args, tensors):
    """Calls the C function on `stream` (the current stream of GPU `dev` when None);
    `tensors` are those that the kernels touch."""
    if stream is not None and stream.device_index != dev:
        raise ValueError(f"stream: expected one of GPU {dev}, got one of GPU {stream.device_index}")
    f = _functions.get(where)
    if f is None:
        f = _functions[where] = getattr(lib(), where)
    if dev != torch.cuda.current_device():
        with torch.cuda.device(dev):
            return _run(where, dev, stream, args, tensors)
    current = torch._C._cuda_getCurrentRawStream(dev)
    if stream is None or stream.cuda_stream == current:
        rc = f(*args, current)
    else:
        rc = f(*args, stream.cuda_stream)
        for t in tensors:
            for x in ((t.codes, t.scales) if type(t) is Mx4 else (t,)):
                if x is not None:
                    x.record_stream(stream)
    if rc != ZO_OK:
        detail = lib().zo_ops_last_hip_error().decode() if rc == ZO_EHIP else ""
        raise ZoError(rc, where, detail)


def zo_mx4_quantize(x, q=None, qt=None, stream=None):
    """x [rows, cols] into q (an Mx4 of rows x cols, blocks along x's rows) and / or
    qt (cols x rows, blocks along x's columns), reading x once."""
    dev = _device_of(x, "x")
    p, dt, ld = _matrix(x, "x", dev)
    rows, cols = x.shape
    _run("zo_mx4_quantize", dev, stream,
         (p, dt, rows, cols, ld, None if q is None else _mx4(q, "q", dev),
          None if qt is None else _mx4(qt, "qt", dev)), (x, q, qt))


def zo_mx4_dequantize(q, out, stream=None):
    """The values of q into out [q.rows, q.cols]."""
    dev = _device_of(out, "out")
    pq = _mx4(q, "q", dev)
    p, dt, ld = _matrix(out, "out", dev, q.rows, q.cols)
    _run("zo_mx4_dequantize", dev, stream, (pq, p, dt, ld), (q, out))


def zo_mx4_product(a, b, out, stream=None):
    """out [a.rows, b.rows] = a b^T, reduced over the columns of both."""
    dev = _device_of(out, "out")
    pa, pb = _mx4(a, "a", dev), _mx4(b, "b", dev)
    p, dt, ld = _matrix(out, "out", dev, a.rows, b.rows)
    _run("zo_mx4_product", dev, stream, (pa, pb, p, dt, ld), (a, b, out))


def zo_mx4_linear(x, w, out, xq, stream=None):
    """out [rows, w.rows] = x quantised along its rows times w^T; xq (an Mx4 of
    x's shape) is workspace."""
    dev = _device_of(x, "x")
    pw, pq = _mx4(w, "w", dev), _mx4(xq, "xq", dev)
    px, dx, ldx = _matrix(x, "x", dev, xq.rows, xq.cols)
    po, do, ldo = _matrix(out, "out", dev, xq.rows, w.rows)
    _run("zo_mx4_linear", dev, stream, (px, dx, ldx, pw, pq, po, do, ldo), (x, w, out, xq))


def zo_top_logits(z, values, columns, lse=None, *, tau=1.0, stream=None):
    """The values.shape[1] largest logits of every row of z [rows, vocab] in
    descending order (ties: lowest column first) into values (float32), their
    columns into columns (int32), and log sum exp(z / tau) into lse [rows]."""
    dev = _device_of(z, "z")
    p, dt, ld = _matrix(z, "z", dev)
    rows, vocab = z.shape
    if values.dim() != 2:
        raise ValueError("values: expected a matrix")
    top = values.shape[1]
    pv = _vector(values, "values", dev, torch.float32, (rows, top))
    pc = _vector(columns, "columns", dev, torch.int32, (rows, top))
    pl = _vector(lse, "lse", dev, torch.float32, (rows,))
    _run("zo_top_logits", dev, stream, (p, dt, rows, vocab, ld, top, float(tau), pv, pc, pl),
         (z, values, columns, lse))


def zo_distill_loss(z, values, columns, loss=None, dz=None, *, tau=1.0, teacher_lse=None,
                    labels=None, kd_weight=1.0, ce_weight=0.0, row_weight=None, stream=None):
    """Distillation from a teacher's top logits: the loss of every row of the
    student's logits z [rows, vocab] into loss (float32 [rows]) and / or its
    gradient into dz (z's type and shape; may be z itself).

    values (float32) and columns (int32), [rows, top], are the teacher's; a
    column outside the vocabulary marks an unused slot.  teacher_lse adds the
    rest of the teacher's mass as one outcome.  labels (int32 [rows], outside
    the vocabulary: none) enter with ce_weight; row_weight (float32 [rows]) is
    the gradient from above, rows of weight 0 are skipped."""
    dev = _device_of(z, "z")
    p, dt, ldz = _matrix(z, "z", dev)
    rows, vocab = z.shape
    if values.dim() != 2:
        raise ValueError("values: expected a matrix")
    top = values.shape[1]
    pdz, lddz = None, 0
    if dz is not None:
        if dz.dtype != z.dtype:
            raise ValueError(f"dz: expected {z.dtype}, got {dz.dtype}")
        pdz, _, lddz = _matrix(dz, "dz", dev, rows, vocab)
    a = _Distill(p, dt, rows, vocab, ldz, top,
                 _vector(values, "values", dev, torch.float32, (rows, top)),
                 _vector(columns, "columns", dev, torch.int32, (rows, top)),
                 _vector(teacher_lse, "teacher_lse", dev, torch.float32, (rows,)),
                 _vector(labels, "labels", dev, torch.int32, (rows,)),
                 _vector(row_weight, "row_weight", dev, torch.float32, (rows,)),
                 float(tau), float(kd_weight), float(ce_weight),
                 _vector(loss, "loss", dev, torch.float32, (rows,)), pdz, lddz)
    _run("zo_distill_loss", dev, stream, (ctypes.byref(a),),
         (z, values, columns, teacher_lse, labels, row_weight, loss, dz))
