"""ctypes binding of include/layers/lsgd_layers.h: the ends of the step's
buffers in a language model. Argument marshalling only, as in _lib.

``embed_lookup``, ``embed_grad``, ``quant8``, ``copy_out8``, ``matmul8`` and
``weight_grad8`` mirror the C entry points (each tries the extension _marshal
first, as _lib's calls do); ``empty8`` allocates an 8-bit
matrix: codes (float8_e4m3fn, rows by pitch8(cols)) and scales (float8_e8m0fnu,
ceil(rows/block) by scale_pitch8(cols)). uint8 tensors of the same bytes do too.
"""
import ctypes
import math

import torch

from . import _lib
from ._lib import (_common_dtype, _dev_tensor, _dtype_code, _native_target, _on, _stream, check, lib, ptr_array)

EXPORTS = ("lsgd_embed_lookup", "lsgd_embed_grad_workspace_size", "lsgd_embed_grad", "lsgd_pitch8",
           "lsgd_scale_pitch8", "lsgd_quant8", "lsgd_copy_out8", "lsgd_matmul8",
           "lsgd_weight_grad8_workspace_size", "lsgd_weight_grad8")

_P, _i32, _i64, _f32, _size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
_int = ctypes.c_int
for _name, _args in {
        "lsgd_embed_lookup": [_P, _int, _i64, _i64, _P, _int, _i64, _f32, _P, _int, _P],
        "lsgd_embed_grad_workspace_size": [_i32, _i64, _i64, _i64, ctypes.POINTER(_size)],
        "lsgd_embed_grad": [_P, _int, _P, _int, _i32, _i64, _i64, _i64, _f32, _P, _int, _i32, _P, _size, _P],
        "lsgd_quant8": [_P, _int, _i64, _i64, _P, _P, _P],
        "lsgd_copy_out8": [_P, _i64, _i64, _P, _P, _i32, _P, _P, _i32, _P],
        "lsgd_matmul8": [_P, _P, _i32, _i64, _P, _P, _i32, _i64, _i64, _P, _int, _P],
        "lsgd_weight_grad8_workspace_size": [_i64, _i64, _i64, ctypes.POINTER(_size)],
        "lsgd_weight_grad8": [_P, _P, _P, _i64, _i64, _i64, _P, _int, _i32, _P, _size, _P]}.items():
    getattr(lib, _name).argtypes, getattr(lib, _name).restype = _args, _int
for _name in ("lsgd_pitch8", "lsgd_scale_pitch8"):
    getattr(lib, _name).argtypes, getattr(lib, _name).restype = [_i64], _i64

_CODES = (torch.float8_e4m3fn, torch.uint8)
_SCALES = (torch.float8_e8m0fnu, torch.uint8)


def pitch8(cols):
    """Bytes from one row of codes to the next: cols rounded up to a multiple of 128."""
    return -(-cols // 128) * 128


def scale_pitch8(cols):
    """Bytes from one row of scales to the next: a byte per 128 columns, a multiple of 4."""
    return -(-cols // 512) * 4


def empty8(rows, cols, block=1, device="cuda"):
    """Uninitialised (codes, scales) of a rows by cols matrix in 8 bits, one
    scale for each `block` rows (1 or 128) by 128 columns."""
    if block not in (1, 128):
        raise ValueError("block must be 1 or 128")
    return (torch.empty(rows, pitch8(cols), device=device, dtype=torch.float8_e4m3fn),
            torch.empty(-(-rows // block), scale_pitch8(cols), device=device, dtype=torch.float8_e8m0fnu))


def _index_code(t, what):
    if t.dtype == torch.int32:
        return 0
    if t.dtype == torch.int64:
        return 1
    raise TypeError("%s must be int32 or int64, got %s" % (what, t.dtype))


def _bytes8(t, what, types, numel, device):
    _dev_tensor(t, what, None, None, device)
    if t.dtype not in types:
        raise TypeError("%s must be %s or %s, got %s" % (what, *types, t.dtype))
    if t.numel() != numel:
        raise ValueError("%s has %d bytes, expected %d" % (what, t.numel(), numel))
    return t.data_ptr()


def _matrix(t, what, dtype=None, device=None):
    """(rows, cols) of a contiguous GPU tensor seen as a matrix of its last dimension."""
    _dev_tensor(t, what, dtype, None, device)
    if t.dim() < 1:
        raise ValueError("%s must have at least one dimension" % what)
    return math.prod(t.shape[:-1]), t.shape[-1]


def _workspace(size_of, sizes, workspace, stream, device):
    """(pointer, bytes, tensor) of the caller's workspace or of a new one."""
    n = ctypes.c_size_t()
    check(size_of(*sizes, ctypes.byref(n)))
    if workspace is not None:
        _dev_tensor(workspace, "workspace", torch.uint8, None, device)
    elif n.value:
        # on the call's stream: memory freed on another may still be read there
        with torch.cuda.stream(stream):
            workspace = torch.empty(n.value, dtype=torch.uint8, device=device)
    else:
        return None, 0, None
    return workspace.data_ptr(), workspace.numel(), workspace


def embed_lookup(table, tokens, out, scale=1.0, stream=None):
    """lsgd_embed_lookup: out[i] = scale * table[tokens[i]], 0 for a token
    outside the table. table: rows by dim (float32 or bfloat16); tokens: int32
    or int64, any shape; out: tokens.numel() by dim elements (float32 or bfloat16)."""
    target = _native_target(table, stream)
    if target is not None:
        st = _lib._marshal.embed_lookup(table, tokens, out, scale, *target)
        if st is not None:
            return check(st)
    rows, dim = _matrix(table, "table")
    dev = table.device
    _dev_tensor(tokens, "tokens", None, None, dev)
    n = tokens.numel()
    _dev_tensor(out, "out", None, n * dim, dev)
    tdt, odt, it = _dtype_code(table, "table"), _dtype_code(out, "out"), _index_code(tokens, "tokens")
    with _on(dev.index):
        st = lib.lsgd_embed_lookup(table.data_ptr(), tdt, rows, dim, tokens.data_ptr(), it, n, scale, out.data_ptr(),
                                   odt, _stream(stream, dev))
    check(st)


def embed_grad_workspace_size(n_workers, n_tokens, rows, dim):
    """Bytes of device workspace that embed_grad needs."""
    n = ctypes.c_size_t()
    check(lib.lsgd_embed_grad_workspace_size(n_workers, n_tokens, rows, dim, ctypes.byref(n)))
    return n.value


def embed_grad(grads, tokens, out, scale=1.0, accumulate=False, workspace=None, stream=None):
    """lsgd_embed_grad: out[v] = scale * the sum of every worker's gradient rows
    whose token is v (+ out[v] with accumulate). grads: a list of tensors, one
    per worker, of n by dim elements (all float32 or all bfloat16); tokens: as
    many tensors of n elements (all int32 or all int64); out: rows by dim
    (float32 or bfloat16). workspace: a uint8 device tensor of
    embed_grad_workspace_size() bytes, 256-byte aligned; by default one is
    allocated for the call."""
    target = _native_target(out, stream)
    if target is not None and workspace is None and stream is None:
        st = _lib._marshal.embed_grad(grads, tokens, out, scale, 1 if accumulate else 0, *target)
        if st is not None:
            return check(st)
    rows, dim = _matrix(out, "out")
    dev = out.device
    if not grads or len(tokens) != len(grads):
        raise ValueError("need as many token tensors as gradients, at least one of each")
    n = tokens[0].numel() if isinstance(tokens[0], torch.Tensor) else 0
    for g, t in zip(grads, tokens):
        _dev_tensor(t, "tokens", None, n, dev)
        _dev_tensor(g, "grad", None, n * dim, dev)
    it = _index_code(tokens[0], "tokens")
    if any(t.dtype != tokens[0].dtype for t in tokens):
        raise TypeError("all tokens must share one dtype")
    gdt, odt = _common_dtype(grads, "grads"), _dtype_code(out, "out")
    with _on(dev.index):
        ws, size, keep = _workspace(lib.lsgd_embed_grad_workspace_size, (len(grads), n, rows, dim), workspace, stream,
                                    dev)
        st = lib.lsgd_embed_grad(ptr_array([g.data_ptr() for g in grads]), gdt,
                                 ptr_array([t.data_ptr() for t in tokens]), it, len(grads), n, rows, dim, scale,
                                 out.data_ptr(), odt, 1 if accumulate else 0, ws, size, _stream(stream, dev))
    check(st)


def quant8(x, codes, scales, stream=None):
    """lsgd_quant8: x (float32 or bfloat16, rows by cols of its last dimension)
    in 8 bits, a scale per row and 128 columns. codes, scales: as empty8(rows, cols)."""
    target = _native_target(x, stream)
    if target is not None:
        st = _lib._marshal.quant8(x, codes, scales, *target)
        if st is not None:
            return check(st)
    rows, cols = _matrix(x, "x")
    dev = x.device
    q = _bytes8(codes, "codes", _CODES, rows * pitch8(cols), dev)
    s = _bytes8(scales, "scales", _SCALES, rows * scale_pitch8(cols), dev)
    xdt = _dtype_code(x, "x")
    with _on(dev.index):
        st = lib.lsgd_quant8(x.data_ptr(), xdt, rows, cols, q, s, _stream(stream, dev))
    check(st)


def copy_out8(params, replicas=(), transposed=(), stream=None):
    """lsgd_copy_out8: every replica = params (float32, rows by cols) in 8 bits,
    a scale per 128 rows and 128 columns; every one of `transposed` = its
    transpose. replicas, transposed: lists of (codes, scales) as empty8(rows,
    cols, 128) and empty8(cols, rows, 128)."""
    target = _native_target(params, stream)
    if target is not None:
        st = _lib._marshal.copy_out8(params, replicas, transposed, *target)
        if st is not None:
            return check(st)
    rows, cols = _matrix(params, "params", torch.float32)
    dev = params.device
    arrays = []
    for copies, r, c, what in ((replicas, rows, cols, "replica"), (transposed, cols, rows, "transposed replica")):
        arrays.append(ptr_array([_bytes8(q, what + " codes", _CODES, r * pitch8(c), dev) for q, _ in copies]))
        arrays.append(ptr_array([_bytes8(s, what + " scales", _SCALES, -(-r // 128) * scale_pitch8(c), dev)
                                 for _, s in copies]))
    with _on(dev.index):
        st = lib.lsgd_copy_out8(params.data_ptr(), rows, cols, arrays[0], arrays[1], len(replicas), arrays[2],
                                arrays[3], len(transposed), _stream(stream, dev))
    check(st)


def _operand8(codes, scales, what, device=None):
    """(codes pointer, scales pointer, block, rows, pitch) of an 8-bit matrix."""
    _dev_tensor(codes, what, None, None, device)
    _dev_tensor(scales, what + " scales", None, None, device or codes.device)
    if codes.dtype not in _CODES or scales.dtype not in _SCALES:
        raise TypeError("%s must be %s with scales %s (or uint8), got %s and %s"
                        % (what, _CODES[0], _SCALES[0], codes.dtype, scales.dtype))
    rows, pitch = _matrix(codes, what)
    if pitch % 128:
        raise ValueError("%s has rows of %d codes, not a multiple of 128" % (what, pitch))
    n, sp = scales.numel(), scale_pitch8(pitch)
    if n == rows * sp:
        block = 1
    elif n == -(-rows // 128) * sp:
        block = 128
    else:
        raise ValueError("%s has %d scales, expected %d by 1 or %d by 128 rows" % (what, n, rows * sp, -(-rows // 128) * sp))
    return codes.data_ptr(), scales.data_ptr(), block, rows, pitch


def matmul8(a, a_scales, b, b_scales, out, stream=None):
    """lsgd_matmul8: out[i][j] = sum over c of a[i][c] * b[j][c], for 8-bit
    matrices a (m rows) and b (n rows) of the same pitch (block 1 or 128, by
    their scales' number); out: m by n, float32 or bfloat16 (exact products and
    float32 sums for both)."""
    target = _native_target(a, stream)
    if target is not None:
        st = _lib._marshal.matmul8(a, a_scales, b, b_scales, out, *target)
        if st is not None:
            return check(st)
    pa, sa, ba, m, pitch = _operand8(a, a_scales, "a")
    dev = a.device
    pb, sb, bb, n, pitch_b = _operand8(b, b_scales, "b", dev)
    if pitch != pitch_b:
        raise ValueError("a has rows of %d codes, b of %d" % (pitch, pitch_b))
    _dev_tensor(out, "out", None, m * n, dev)
    odt = _dtype_code(out, "out")
    with _on(dev.index):
        st = lib.lsgd_matmul8(pa, sa, ba, m, pb, sb, bb, n, pitch, out.data_ptr(), odt, _stream(stream, dev))
    check(st)


def weight_grad8_workspace_size(m, n, k):
    """Bytes of device workspace that weight_grad8 needs (0 for many sizes)."""
    b = ctypes.c_size_t()
    check(lib.lsgd_weight_grad8_workspace_size(m, n, k, ctypes.byref(b)))
    return b.value


def weight_grad8(grad, x, x_scales, out, accumulate=False, workspace=None, stream=None):
    """lsgd_weight_grad8: out[j][c] = sum over i of grad[i][j] * x[i][c] (+
    out[j][c] with accumulate). grad: m by n, bfloat16; x: m by k in 8 bits, a
    scale per row and 128 columns (as quant8 writes it); out: n by k, float32
    or bfloat16. workspace: as embed_grad's, of weight_grad8_workspace_size() bytes."""
    target = _native_target(out, stream)
    if target is not None and workspace is None and stream is None:
        st = _lib._marshal.weight_grad8(grad, x, x_scales, out, 1 if accumulate else 0, *target)
        if st is not None:
            return check(st)
    n, k = _matrix(out, "out")
    dev = out.device
    m, gn = _matrix(grad, "grad", torch.bfloat16, dev)
    if gn != n:
        raise ValueError("grad has %d columns, out %d rows" % (gn, n))
    q = _bytes8(x, "x", _CODES, m * pitch8(k), dev)
    s = _bytes8(x_scales, "x_scales", _SCALES, m * scale_pitch8(k), dev)
    odt = _dtype_code(out, "out")
    with _on(dev.index):
        ws, size, keep = _workspace(lib.lsgd_weight_grad8_workspace_size, (m, n, k), workspace, stream, dev)
        st = lib.lsgd_weight_grad8(grad.data_ptr(), q, s, m, n, k, out.data_ptr(), odt, 1 if accumulate else 0, ws,
                                   size, _stream(stream, dev))
    check(st)
