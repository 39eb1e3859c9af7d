"""Binding of the operators that write a paged KV cache and that hold it in 4 bits (include/ibp.h,
ibp_kv_append, ibp_kv4_* and ibp_attn_decode4).

Argument marshalling only, on GPU tensors as in attention.py. A 4-bit cache's pools are torch.uint8,
[n_pages][kv_heads][page_tokens][ibp_kv4_record(head_dim)] (strides but the last are free, multiples of
16); ibp_kv_evict takes them as pool.view(torch.bfloat16).
"""
import ctypes
import struct

import torch

from . import _check as check
from . import lib
from .attention import (TYPES, _array, _count, _device, _rows, _space, _stream, _tensor, _u32, _u64, _vp, ibp_attn,
                        ibp_pages, ibp_rows)


class ibp_rotation(ctypes.Structure):
    _fields_ = [("d_table", _vp), ("positions", _u64), ("turned", _u32), ("halves", _u32)]


_p = ctypes.POINTER
_append = [_p(ibp_attn), _p(ibp_rows), _p(ibp_rows), _p(ibp_rows), _p(ibp_rows), _p(ibp_rotation), _vp, _u32, _p(ibp_pages),
           _vp, _vp, _vp, _vp, _u64, _vp]
SIGS = {
    "ibp_kv_append": _append,
    "ibp_kv4_record": [_u32, _p(_u32)],
    "ibp_kv4_append": _append,
    "ibp_kv4_read": [_p(ibp_attn), _p(ibp_pages), _vp, _u32, _vp, _vp, _p(ibp_rows), _p(ibp_rows), _vp],
    "ibp_attn_decode4_workspace": [_u32, _u32, _u32, _u32, _u32, ctypes.c_int, _p(_u64)],
    "ibp_attn_decode4": [_p(ibp_attn), _p(ibp_rows), _p(ibp_pages), _vp, _u32, _p(ibp_rows), _vp, _vp, _u64, _vp, _u64, _vp],
}

for _f, _args in SIGS.items():
    getattr(lib(), _f).argtypes = _args
    getattr(lib(), _f).restype = ctypes.c_int

# A step of a serving loop is a few microseconds on the GPU, and a call's checks and arguments count beside that: what is in order
# is passed at once, and the rest left to the functions that say what is wrong; the structures are packed
# into bytes, whose addresses the calls below take.


def _taking(name):
    """The library's function of that name, its structures passed as bytes."""
    args = [_vp if hasattr(x, "contents") else x for x in SIGS[name]]
    return ctypes.CFUNCTYPE(ctypes.c_int, *args)((name, lib()))


_KV_APPEND, _KV4_APPEND, _KV4_READ, _DECODE4 = (_taking(f) for f in ("ibp_kv_append", "ibp_kv4_append", "ibp_kv4_read", "ibp_attn_decode4"))
_pack_attn, _pack_rows, _pack_pages, _pack_rotation = (struct.Struct(x).pack for x in ("4IfI", "4Q", "3Q2I7Q", "2Q2I"))
assert all(struct.calcsize(x) == ctypes.sizeof(y) for x, y in (("4IfI", ibp_attn), ("4Q", ibp_rows), ("3Q2I7Q", ibp_pages), ("2Q2I", ibp_rotation)))
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
if _raw_stream is None:                              # (a torch that has no handles without Stream objects around them)
    def _raw_stream(device):
        return torch.cuda.current_stream(device).cuda_stream


def _beyond(what, *sizes):
    return ValueError(f"{what} must fit 32 bits, not {', '.join(str(x) for x in sizes)}")


def _device_of(x, what):
    try:
        device = x.get_device()                      # (-1 for a host tensor)
        if device >= 0 and device == torch._C._cuda_getDevice():
            return device
    except AttributeError:
        pass
    return _device(x, what)


def _rows_of(x, what, kind, device, heads=None, dim=None):
    try:
        if x.dtype is kind and x.get_device() == device:
            n, h, d = x.shape
            a, b, c = x.stride()
            if c == 1 and (heads is None or h == heads) and (dim is None or d == dim):
                return _pack_rows(x.data_ptr(), n, a if n > 1 else 0, b if h > 1 else 0)
    except (AttributeError, ValueError):             # (not a tensor, not of three dimensions)
        pass
    return bytes(_rows(x, what, kind, device, heads, dim))


def _numbers(x, what, kind, device, shape):
    """Address of a contiguous tensor of one type and shape."""
    try:
        if x.dtype is kind and x.get_device() == device and x.shape == shape and x.is_contiguous():
            return x.data_ptr()
    except AttributeError:
        pass
    return _array(x, what, kind, device, shape)


def _pool_of(keys, values, table, device, kind, unit, kv_heads, width, what):
    """Pools [n_pages][kv_heads][page_tokens][width] of one kind (unit: elements of it in 2 bytes) with their table: its sequences,
    and the pages."""
    try:
        shape = keys.shape
        n, h, t, w = shape
        if (keys.dtype is not kind or values.dtype is not kind or keys.get_device() != device or values.get_device() != device
                or values.shape != shape or h != kv_heads or w != width):
            raise ValueError
        a, b, c, d = keys.stride()
        e, f, g, i = values.stride()
    except (AttributeError, ValueError):
        _wrong_pools(keys, values, device, kind, kv_heads, width, what)
    if d != 1 or i != 1:
        raise TypeError("keys and values: the last dimension must be contiguous")
    if n == 1 or h == 1 or t == 1:                   # (a dimension of one has no stride)
        a, e = (a, e) if n > 1 else (0, 0)
        b, f = (b, f) if h > 1 else (0, 0)
        c, g = (c, g) if t > 1 else (0, 0)
    if (a | b | c | e | f | g) & (8 * unit - 1):
        raise ValueError("keys and values: strides must be multiples of 16 bytes")
    try:
        sequences, pages = table.shape
        if table.dtype is not torch.int32 or table.get_device() != device or not table.is_contiguous():
            raise ValueError
    except (AttributeError, ValueError):
        _array(table, "table", torch.int32, device)
        raise ValueError("table must be [sequences][pages]") from None
    if unit == 2:
        a, b, c, e, f, g = a >> 1, b >> 1, c >> 1, e >> 1, f >> 1, g >> 1
    try:
        return sequences, _pack_pages(keys.data_ptr(), values.data_ptr(), n, t, pages, table.data_ptr(), a, b, c, e, f, g)
    except struct.error:
        raise _beyond("slots of a page and pages of a sequence", t, pages) from None


def _wrong_pools(keys, values, device, kind, kv_heads, width, what):
    for x, name in ((keys, "keys"), (values, "values")):
        _tensor(x, name, device)
        if x.dtype != kind:
            raise TypeError(f"{name} must be {kind}, not {x.dtype}")
        if x.dim() != 4 or x.shape[1] != kv_heads or x.shape[3] != width:
            raise ValueError(f"{name} must be [n_pages][{kv_heads}][page_tokens][{width}] ({what}), not {list(x.shape)}")
    raise ValueError("keys and values must have the same shape")


def _sequences(n, lens, starts, rows, device):
    """The addresses of n sequences' lengths and starts."""
    if n >> 32:
        raise _beyond("sequences", n)
    lens_at = _numbers(lens, "lens", torch.int32, device, (n,))
    if starts is None:
        if rows != n:
            raise ValueError("without starts every sequence has one row")
        return lens_at, None
    return lens_at, _numbers(starts, "starts", torch.int32, device, (n + 1,))


def _appender(call, name, four, about):
    def append(k, v, keys, values, table, lens, next_positions, starts=None, rotation=None, halves=True, q=None, q_out=None, weights=None,
               positions=None, stream=None):
        device = _device_of(k, "k")
        kind = k.dtype
        if kind not in TYPES:
            raise TypeError(f"k must be bfloat16 or float16, not {kind}")
        rk = _rows_of(k, "k", kind, device)
        rows, kv_heads, dim = k.shape
        rv = _rows_of(v, "v", kind, device, kv_heads, dim)
        if four:
            n, pages = _pool_of(keys, values, table, device, torch.uint8, 2, kv_heads, ibp_kv4_record(dim), "records")
        else:
            n, pages = _pool_of(keys, values, table, device, kind, 1, kv_heads, dim, "values")
        lens_at, starts_at = _sequences(n, lens, starts, rows, device)
        next_at = lens_at if next_positions is lens else _numbers(next_positions, "next_positions", torch.int32, device, (n,))
        rq = ro = turn = None
        heads = kv_heads
        if q is not None:
            rq = _rows_of(q, "q", kind, device, None, dim)
            heads = q.shape[1]
            ro = rq if q_out is None or q_out is q else _rows_of(q_out, "q_out", kind, device, heads, dim)
        elif q_out is not None:
            raise ValueError("q_out without q")
        if rotation is not None:
            shape = rotation.shape if isinstance(rotation, torch.Tensor) else ()
            at = _numbers(rotation, "rotation", torch.float32, device, shape)
            if len(shape) != 3 or shape[2] != 2:
                raise ValueError("rotation must be [positions][pairs][2]")
            try:
                turn = _pack_rotation(at, shape[0], 2 * shape[1], 1 if halves else 0)
            except struct.error:
                raise _beyond("values that a rotation turns", 2 * shape[1]) from None
        slots, weights_at, positions_at = 0, None, None
        if weights is not None:
            weights_at, slots = _tracked(weights, "weights", torch.float32, device, n, kv_heads, None)
        if positions is not None:
            positions_at, slots = _tracked(positions, "positions", torch.int32, device, n, kv_heads, slots if weights is not None else None)
        try:
            a = _pack_attn(TYPES[kind], heads, kv_heads, dim, 1.0, 0)
        except struct.error:
            raise _beyond("heads and head_dim", heads, kv_heads, dim) from None
        status = call(a, rk, rv, rq, ro, turn, starts_at, n, pages, lens_at, next_at, weights_at, positions_at,
                      slots, _raw_stream(device) if stream is None else _stream(stream, device))
        if status:
            check(status, name)

    append.__name__ = append.__qualname__ = name
    append.__doc__ = about
    return append


def _tracked(x, what, kind, device, n, kv_heads, slots):
    shape = x.shape if isinstance(x, torch.Tensor) else ()
    at = _numbers(x, what, kind, device, shape)
    if len(shape) != 3 or shape[0] != n or shape[1] != kv_heads or (slots is not None and shape[2] != slots):
        raise ValueError("weights and positions must be [sequences][kv_heads][slots]")
    return at, shape[2]


_records = {}


def ibp_kv4_record(head_dim):
    """Bytes of one token's key or value of one head in a 4-bit cache."""
    got = _records.get(head_dim)
    if got is None:
        out = _u32(0)
        check(lib().ibp_kv4_record(_count(head_dim, "head_dim"), out), "ibp_kv4_record")
        got = _records[head_dim] = out.value
    return got


ibp_kv_append = _appender(_KV_APPEND, "ibp_kv_append", False, """Rows of k and v [rows][kv_heads][dim] become the last slots of their sequences in the pools keys and
    values [n_pages][kv_heads][page_tokens][dim], keys turned by their positions. starts (int32
    [sequences + 1]): where each sequence's rows begin; None: one row each. lens and next_positions (int32)
    are those after the call, and may be one tensor. rotation: float32 [positions][pairs][2], cosine and sine;
    halves: pairs are (i, i + pairs), else (2 i, 2 i + 1). q [rows][q_heads][dim] is turned into q_out (None: in
    place). weights (float32) and positions (int32) [sequences][kv_heads][slots] get 0 and the position.""")
ibp_kv4_append = _appender(_KV4_APPEND, "ibp_kv4_append", True, """ibp_kv_append into pools of 4-bit records, uint8 [n_pages][kv_heads][page_tokens][ibp_kv4_record(dim)].""")


def ibp_kv4_read(keys, values, table, lens, k, v, starts=None, first=None, stream=None):
    """What the slots of a 4-bit cache stand for, into packed rows k and v [rows][kv_heads][dim]: slot first[s] + i
    (first None: i) of sequence s to row starts[s] + i (starts None: one row each), up to lens[s]."""
    device = _device_of(k, "k")
    kind = k.dtype
    if kind not in TYPES:
        raise TypeError(f"k must be bfloat16 or float16, not {kind}")
    rk = _rows_of(k, "k", kind, device)
    rows, kv_heads, dim = k.shape
    rv = _rows_of(v, "v", kind, device, kv_heads, dim)
    n, pages = _pool_of(keys, values, table, device, torch.uint8, 2, kv_heads, ibp_kv4_record(dim), "records")
    lens_at, starts_at = _sequences(n, lens, starts, rows, device)
    first_at = None if first is None else _numbers(first, "first", torch.int32, device, (n,))
    try:
        a = _pack_attn(TYPES[kind], kv_heads, kv_heads, dim, 1.0, 0)
    except struct.error:
        raise _beyond("heads and head_dim", kv_heads, dim) from None
    status = _KV4_READ(a, pages, lens_at, n, starts_at, first_at, rk, rv,
                       _raw_stream(device) if stream is None else _stream(stream, device))
    if status:
        check(status, "ibp_kv4_read")


def ibp_attn_decode4_workspace(n_seqs, q_heads, kv_heads, head_dim, max_len, weights):
    out = _u64(0)
    check(lib().ibp_attn_decode4_workspace(_count(n_seqs, "n_seqs"), _count(q_heads, "q_heads"), _count(kv_heads, "kv_heads"),
                                           _count(head_dim, "head_dim"), _count(max_len, "max_len"), int(bool(weights)), out),
          "ibp_attn_decode4_workspace")
    return out.value


def ibp_attn_decode4(q, keys, values, table, lens, max_len, out, lse=None, weights=None, scale=None, workspace=None, stream=None):
    """ibp_attn_decode over a cache of 4-bit records: q and out [sequences][q_heads][dim], the rest as there."""
    device = _device_of(q, "q")
    if q.dtype not in TYPES:
        raise TypeError(f"q must be bfloat16 or float16, not {q.dtype}")
    rq = _rows_of(q, "q", q.dtype, device)
    n, heads, dim = q.shape
    _tensor(keys, "keys", device)
    kv_heads = keys.shape[1] if keys.dim() == 4 else 0
    sequences, pages = _pool_of(keys, values, table, device, torch.uint8, 2, kv_heads, ibp_kv4_record(dim), "records")
    if sequences != n:
        raise ValueError("table must have a row for every sequence")
    lens_at = _numbers(lens, "lens", torch.int32, device, (n,))
    ro = _rows_of(out, "out", q.dtype, device, heads, dim)
    lse_at = None if lse is None else _numbers(lse, "lse", torch.float32, device, (n, heads))
    weights_at, slots = None, 0
    if weights is not None:
        weights_at, slots = _tracked(weights, "weights", torch.float32, device, n, kv_heads, None)
    scale = dim ** -0.5 if scale is None else max(min(scale, 3e38), -3e38)       # (the library refuses what is too large for it)
    try:
        a = _pack_attn(TYPES[q.dtype], heads, kv_heads, dim, scale, 0)
    except struct.error:
        raise _beyond("heads and head_dim", heads, kv_heads, dim) from None
    need = 0
    if workspace is None:
        need = ibp_attn_decode4_workspace(n, heads, kv_heads, dim, max_len, weights is not None)
    at, size, held = _space(workspace, need, device, stream)
    status = _DECODE4(a, rq, pages, lens_at, _count(max_len, "max_len"), ro, lse_at, weights_at, slots, at, size,
                      _raw_stream(device) if stream is None else _stream(stream, device))
    if status:
        check(status, "ibp_attn_decode4")
