"""Python binding of the operators declared in ``include/zo_ops.h``.

Argument marshalling only, with the C names: matrices in microscaled 4-bit
floating point (``Mx4``) and in 8-bit integers (``I8``) and their products, the
root-mean-square norm, a teacher's top logits, the distillation loss with the
gradient of the student's logits, the log probabilities of tokens.  Device buffers
are torch tensors; two-dimensional ones may have any row stride as long as
their rows are contiguous.  Every call checks element types, shapes and
devices before anything reaches the device and enqueues on ``stream`` (torch's
current stream by default).  On another stream than the current one the
tensors are recorded as in use there; ordering the streams stays with the
caller.
"""
import ctypes

import torch

from . import (ZoError, ZO_EHIP, ZO_EINVAL, ZO_OK, _Distill, _I8, _Mx4, _Norm, _NormBack, _Score,
               _ScoreBack, lib)

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


def zo_i8_code_bytes(rows, cols):
    """Bytes of the codes of a rows x cols 8-bit matrix."""
    return _size(lib().zo_i8_code_bytes(int(rows), int(cols)), "zo_i8_code_bytes")


def zo_i8_work_bytes(rows, cols):
    """Bytes of the workspace in which zo_i8_quantize finds the largest magnitudes of the
    columns of a rows x cols matrix."""
    return _size(lib().zo_i8_work_bytes(int(rows), int(cols)), "zo_i8_work_bytes")


class I8:
    """A rows x cols matrix in 8-bit integers with a scale for each row: ``codes``, an
    int8 device tensor of rows of cols rounded up to a multiple of 128 (zero beyond cols),
    and ``scales``, float32 [rows] (allocated when not given).  Its rows are the axis that
    products reduce over."""

    __slots__ = ("rows", "cols", "codes", "scales", "dev", "_c", "_at")

    def __init__(self, rows, cols, codes=None, scales=None, device="cuda"):
        rows, cols = int(rows), int(cols)
        if not (0 <= rows <= _MAX_DIM and 0 <= cols <= _MAX_DIM):
            raise ZoError(ZO_EINVAL, "I8")
        n = rows * ((cols + 127) >> 7 << 7)
        if codes is None:
            codes = torch.empty(n, dtype=torch.int8, device=device)
        if scales is None:
            scales = torch.empty(rows, dtype=torch.float32, device=codes.device)
        if codes.dtype is not torch.int8 or scales.dtype is not torch.float32:
            raise ValueError(f"codes, scales: expected int8 and float32, got {codes.dtype} and "
                             f"{scales.dtype}")
        if codes.numel() < n or not codes.is_contiguous():
            raise ValueError(f"codes: needs {n} contiguous elements, has {codes.numel()}")
        if scales.numel() < rows or not scales.is_contiguous():
            raise ValueError(f"scales: needs {rows} contiguous elements, has {scales.numel()}")
        dev = codes.get_device()
        if dev < 0 or scales.get_device() != dev:
            raise ValueError("codes, scales: expected tensors on one GPU")
        self.rows, self.cols, self.codes, self.scales, self.dev = rows, cols, codes, scales, dev
        self._c = _I8(codes.data_ptr(), scales.data_ptr(), rows, cols)
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


def _i8(q, what, dev):
    """Address of q's C struct."""
    if type(q) is not I8:
        raise ValueError(f"{what}: expected an I8")
    if q.dev != dev:
        raise ValueError(f"{what}: expected an I8 on GPU {dev}, got one on GPU {q.dev}")
    return q._at


def _same(t, what, dev, dtype, rows, cols):
    """(pointer, row stride) of a matrix of this type and shape, or (None, 0) for None."""
    if t is None:
        return None, 0
    if t.dtype is not dtype:
        raise ValueError(f"{what}: expected {dtype}, got {t.dtype}")
    p, _, ld = _matrix(t, what, dev, rows, cols)
    return p, ld


def _weight(t, dev, dtype, cols):
    """(pointer, element type) of a norm's weight."""
    if t.dtype is not dtype and t.dtype is not torch.float32:
        raise ValueError(f"weight: expected {dtype} or float32, got {t.dtype}")
    return _vector(t, "weight", dev, t.dtype, (cols,)), _DTYPES[t.dtype]


def _room(t, what, dev, size):
    """Pointer of a workspace of at least `size` bytes."""
    if not t.is_contiguous() or t.numel() * t.element_size() < size:
        raise ValueError(f"{what}: needs {size} contiguous bytes, has "
                         f"{t.numel() * t.element_size()}")
    return _at(t, what, dev)


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
            for x in ((t.codes, t.scales) if type(t) in (Mx4, I8) else (t,)):
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


def zo_i8_quantize(x, q=None, qt=None, work=None, stream=None):
    """x [rows, cols] into q (an I8 of rows x cols, a scale for each of x's rows) and / or
    qt (cols x rows, a scale for each of x's columns); qt needs work, a tensor of
    zo_i8_work_bytes(rows, cols) bytes."""
    dev = _device_of(x, "x")
    p, dt, ld = _matrix(x, "x", dev)
    rows, cols = x.shape
    room = None
    if qt is not None and rows and cols:
        if work is None:
            raise ValueError("work: needed with qt")
        room = _room(work, "work", dev, lib().zo_i8_work_bytes(rows, cols))
    _run("zo_i8_quantize", dev, stream,
         (p, dt, rows, cols, ld, None if q is None else _i8(q, "q", dev),
          None if qt is None else _i8(qt, "qt", dev), room), (x, q, qt, work))


def zo_i8_dequantize(q, out, stream=None):
    """The values of q into out [q.rows, q.cols]."""
    dev = _device_of(out, "out")
    pq = _i8(q, "q", dev)
    p, dt, ld = _matrix(out, "out", dev, q.rows, q.cols)
    _run("zo_i8_dequantize", dev, stream, (pq, p, dt, ld), (q, out))


def zo_i8_product(a, b, out, stream=None):
    """out [a.rows, b.rows] = a b^T, reduced over the columns of both (at most 131072)."""
    dev = _device_of(out, "out")
    pa, pb = _i8(a, "a", dev), _i8(b, "b", dev)
    p, dt, ld = _matrix(out, "out", dev, a.rows, b.rows)
    _run("zo_i8_product", dev, stream, (pa, pb, p, dt, ld), (a, b, out))


def zo_i8_linear(x, w, out, xq, stream=None):
    """out [rows, w.rows] = x quantised along its rows times w^T; xq (an I8 of x's shape)
    is workspace."""
    dev = _device_of(x, "x")
    pw, pq = _i8(w, "w", dev), _i8(xq, "xq", dev)
    px, dx, ldx = _matrix(x, "x", dev, xq.rows, xq.cols)
    po, do, ldo = _matrix(out, "out", dev, xq.rows, w.rows)
    _run("zo_i8_linear", dev, stream, (px, dx, ldx, pw, pq, po, do, ldo), (x, w, out, xq))


def zo_rms_norm(x, weight, *, residual=None, h=None, out=None, q=None, rstd=None, eps=1e-5,
                stream=None):
    """h = x + residual (x [rows, cols]; without a residual x) and its root-mean-square norm
    times weight (x's type or float32, [cols]): into out (x's type) and / or q (an I8 of
    x's shape); 1 / sqrt(mean h^2 + eps) into rstd (float32 [rows]), which with h is what
    the gradient needs.  h may be x or residual itself, and so may out where h is not."""
    dev = _device_of(x, "x")
    p, dt, ldx = _matrix(x, "x", dev)
    rows, cols = x.shape
    dtype = x.dtype
    pr, ldr = _same(residual, "residual", dev, dtype, rows, cols)
    pw, wt = _weight(weight, dev, dtype, cols)
    ph, ldh = _same(h, "h", dev, dtype, rows, cols)
    po, ldo = _same(out, "out", dev, dtype, rows, cols)
    a = _Norm(p, dt, rows, cols, ldx, pr, ldr, pw, wt, float(eps), ph, ldh, po, ldo,
              None if q is None else _i8(q, "q", dev),
              _vector(rstd, "rstd", dev, torch.float32, (rows,)))
    _run("zo_rms_norm", dev, stream, (ctypes.byref(a),), (x, residual, weight, h, out, q, rstd))


def zo_rms_norm_work_bytes(rows, cols):
    """Bytes of the workspace in which zo_rms_norm_grad sums the gradient of the weight."""
    return _size(lib().zo_rms_norm_work_bytes(int(rows), int(cols)), "zo_rms_norm_work_bytes")


def zo_rms_norm_grad(dy, h, weight, rstd, dx=None, dw=None, *, dh=None, work=None, stream=None):
    """The gradients of zo_rms_norm from dy, that of out: dx (of x and of the residual; dh,
    what reaches h past the norm, is added) and dw (float32 [cols]), which needs work, a
    tensor of zo_rms_norm_work_bytes(rows, cols) bytes.  dx may be dy, h or dh itself."""
    dev = _device_of(dy, "dy")
    p, dt, lddy = _matrix(dy, "dy", dev)
    rows, cols = dy.shape
    dtype = dy.dtype
    ph, ldh = _same(h, "h", dev, dtype, rows, cols)
    pw, wt = _weight(weight, dev, dtype, cols)
    po, lddh = _same(dh, "dh", dev, dtype, rows, cols)
    px, lddx = _same(dx, "dx", dev, dtype, rows, cols)
    room = None
    if dw is not None and rows:
        if work is None:
            raise ValueError("work: needed with dw")
        room = _room(work, "work", dev, lib().zo_rms_norm_work_bytes(rows, cols))
    a = _NormBack(p, dt, rows, cols, lddy, ph, ldh, pw, wt,
                  _vector(rstd, "rstd", dev, torch.float32, (rows,)), po, lddh, px, lddx,
                  _vector(dw, "dw", dev, torch.float32, (cols,)), room)
    _run("zo_rms_norm_grad", dev, stream, (ctypes.byref(a),),
         (dy, h, weight, rstd, dh, dx, dw, work))


def zo_token_logprobs(z, tokens=None, logp=None, stats=None, values=None, columns=None, *,
                      tau=1.0, stream=None):
    """Under softmax(z / tau) of every row of z [rows, vocab]: the log probability of the
    row's token (tokens int32 [rows], outside the vocabulary: none) into logp (float32
    [rows]); the largest logit, the logarithm of the sum of exponentials about it and the
    entropy into stats (float32 [rows, 3]), which the gradient needs; the values.shape[1]
    largest log probabilities in descending order into values (float32) and their columns
    into columns (int32)."""
    dev = _device_of(z, "z")
    p, dt, ld = _matrix(z, "z", dev)
    rows, vocab = z.shape
    top = 0
    if values is not None:
        if values.dim() != 2 or columns is None:
            raise ValueError("values, columns: expected two matrices")
        top = values.shape[1]
    elif columns is not None:
        raise ValueError("values, columns: expected two matrices")
    if (tokens is None) != (logp is None):
        raise ValueError("tokens, logp: expected both or neither")
    a = _Score(p, dt, rows, vocab, ld, _vector(tokens, "tokens", dev, torch.int32, (rows,)),
               float(tau),
               _vector(logp, "logp", dev, torch.float32, (rows,)),
               _vector(stats, "stats", dev, torch.float32, (rows, 3)), top,
               _vector(values, "values", dev, torch.float32, (rows, top)),
               _vector(columns, "columns", dev, torch.int32, (rows, top)))
    _run("zo_token_logprobs", dev, stream, (ctypes.byref(a),),
         (z, tokens, logp, stats, values, columns))


def zo_token_logprobs_grad(z, stats, dz, *, tokens=None, dlogp=None, dentropy=None, tau=1.0,
                           stream=None):
    """The gradient of z (z's type and shape; may be z itself) from those of the tokens'
    log probabilities and / or of the entropies (float32 [rows]), with the stats of
    zo_token_logprobs.  Rows in which both are 0 are not read."""
    dev = _device_of(z, "z")
    p, dt, ld = _matrix(z, "z", dev)
    rows, vocab = z.shape
    pd, ldd = _same(dz, "dz", dev, z.dtype, rows, vocab)
    a = _ScoreBack(p, dt, rows, vocab, ld, _vector(tokens, "tokens", dev, torch.int32, (rows,)),
                   _vector(stats, "stats", dev, torch.float32, (rows, 3)), float(tau),
                   _vector(dlogp, "dlogp", dev, torch.float32, (rows,)),
                   _vector(dentropy, "dentropy", dev, torch.float32, (rows,)), pd, ldd)
    _run("zo_token_logprobs_grad", dev, stream, (ctypes.byref(a),),
         (z, tokens, stats, dlogp, dentropy, dz))
