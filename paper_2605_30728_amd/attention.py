"""Binding of the attention operators over KV tensors (include/ibp.h, ibp_attn_* and ibp_kv_evict).

Argument marshalling only, on GPU tensors: torch.bfloat16 or torch.float16 values in rows
[rows][heads][head_dim] and pools of pages [n_pages][kv_heads][page_tokens][head_dim], whose last
dimension is contiguous and whose other strides are free (multiples of 8); a pool in
[page][token][head] order is passed as its transposed view. Intermediate results go to `workspace`,
a uint8 tensor of the size that the _workspace call gives; None takes one from torch's allocator
for the call. The operators serve inference: results carry no gradient, whatever their inputs ask for.
"""
import ctypes

import torch

from . import _check as check
from . import lib

IBP_BF16, IBP_F16 = 0, 1
IBP_ATTN_CAUSAL = 1
TYPES = {torch.bfloat16: IBP_BF16, torch.float16: IBP_F16}

_u64, _u32 = ctypes.c_uint64, ctypes.c_uint32


class ibp_attn(ctypes.Structure):
    _fields_ = [("type", _u32), ("q_heads", _u32), ("kv_heads", _u32), ("head_dim", _u32), ("scale", ctypes.c_float),
                ("flags", _u32)]


class ibp_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", _u64), ("row_stride", _u64), ("head_stride", _u64)]


class ibp_pages(ctypes.Structure):
    _fields_ = [("keys", ctypes.c_void_p), ("values", ctypes.c_void_p), ("n_pages", _u64), ("page_tokens", _u32),
                ("table_pages", _u32), ("d_table", ctypes.c_void_p),
                ("key_page_stride", _u64), ("key_head_stride", _u64), ("key_token_stride", _u64),
                ("value_page_stride", _u64), ("value_head_stride", _u64), ("value_token_stride", _u64)]


_p = ctypes.POINTER
_vp = ctypes.c_void_p
SIGS = {
    "ibp_attn_prompt_workspace": [_u32, _u32, _u64, _u64, _u32, _p(_u64)],
    "ibp_attn_prompt": [_p(ibp_attn), _p(ibp_rows), _p(ibp_rows), _p(ibp_rows), _vp, _vp, _u32, _p(ibp_rows), _vp, _vp, _u64, _vp],
    "ibp_attn_key_weights_workspace": [_u32, _u32, _u64, _u32, _p(_u64)],
    "ibp_attn_key_weights": [_p(ibp_attn), _p(ibp_rows), _p(ibp_rows), _vp, _vp, _u32, _vp, _vp, _vp, _u64, _vp],
    "ibp_attn_decode_workspace": [_u32, _u32, _u32, _u32, _u32, ctypes.c_int, _p(_u64)],
    "ibp_attn_decode": [_p(ibp_attn), _p(ibp_rows), _p(ibp_pages), _vp, _u32, _p(ibp_rows), _vp, _vp, _u64, _vp, _u64, _vp],
    "ibp_kv_evict_workspace": [_u32, _u32, _u32, _u32, _p(_u64)],
    "ibp_kv_evict": [_p(ibp_attn), _p(ibp_pages), _vp, _u32, _u32, _u32, _u32, _vp, _vp, _vp, _u64, _vp, _vp, _u64, _vp, _vp,
                     _u64, _vp],
}

for _f, _args in SIGS.items():
    getattr(lib(), _f).argtypes = _args
    getattr(lib(), _f).restype = ctypes.c_int


def _tensor(x, what, device):
    """Checks that x is a tensor on the GPU that the call runs on."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{what} must be a GPU tensor, not {type(x).__name__}")
    if x.get_device() != device:
        raise TypeError(f"{what} must be on the current GPU, not on {x.device}")


def _device(x, what):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise TypeError(f"{what} must be a GPU tensor")
    device = torch.cuda.current_device()
    _tensor(x, what, device)
    return device


def _rows(x, what, kind, device, heads=None, dim=None):
    _tensor(x, what, device)
    if x.dtype != kind:
        raise TypeError(f"{what} must be {kind}, not {x.dtype}")
    if x.dim() != 3:
        raise ValueError(f"{what} must be [rows][heads][head_dim]")
    n, h, d = x.shape
    if (heads is not None and h != heads) or (dim is not None and d != dim):
        raise ValueError(f"{what}: {h} heads of {d}, expected {heads} of {dim}")
    s = x.stride()
    if s[2] != 1 and d != 1:
        raise TypeError(f"{what}: the last dimension must be contiguous")
    return ibp_rows(x.data_ptr(), n, s[0] if n > 1 else 0, s[1] if h > 1 else 0)


def _pages(k, v, table, device):
    for x, what in ((k, "keys"), (v, "values")):
        _tensor(x, what, device)
        if x.dim() != 4:
            raise ValueError(f"{what} must be [n_pages][kv_heads][page_tokens][head_dim]")
        if x.stride(3) != 1 and x.shape[3] != 1:
            raise TypeError(f"{what}: the last dimension must be contiguous")
    if k.dtype not in TYPES or v.dtype != k.dtype:
        raise TypeError(f"keys and values must both be bfloat16 or float16, not {k.dtype} and {v.dtype}")
    if k.shape != v.shape:
        raise ValueError("keys and values must have the same shape")
    _array(table, "table", torch.int32, device)
    if table.dim() != 2:
        raise ValueError("table must be [sequences][pages]")
    n, h, t, _ = k.shape
    one = lambda s: (s[0] if n > 1 else 0, s[1] if h > 1 else 0, s[2] if t > 1 else 0)  # noqa: E731
    return ibp_pages(k.data_ptr(), v.data_ptr(), n, t, table.shape[1], table.data_ptr(), *one(k.stride()), *one(v.stride()))


def _array(x, what, kind, device, shape=None):
    """A contiguous tensor of one type; shape: the least it must have."""
    _tensor(x, what, device)
    if x.dtype != kind:
        raise TypeError(f"{what} must be {kind}, not {x.dtype}")
    if not x.is_contiguous():
        raise TypeError(f"{what} must be contiguous")
    if shape is not None and tuple(x.shape) != shape:
        raise ValueError(f"{what} must be {list(shape)}, not {list(x.shape)}")
    return x.data_ptr()


def _attn(q, kv_heads, dim, scale, causal=False):
    heads = q.shape[1]
    return ibp_attn(TYPES[q.dtype], heads, kv_heads, dim, dim ** -0.5 if scale is None else scale,
                    IBP_ATTN_CAUSAL if causal else 0)


def _starts(q_starts, k_starts, device):
    _array(q_starts, "q_starts", torch.int32, device)
    _array(k_starts, "k_starts", torch.int32, device)
    if q_starts.dim() != 1 or q_starts.shape != k_starts.shape or q_starts.numel() < 1:
        raise ValueError("q_starts and k_starts must each hold one start per sequence and the end")
    return q_starts.numel() - 1


def _space(workspace, need, device, stream):
    """Address and size of the workspace, and what keeps it alive during the call. Memory that is taken here
    belongs to the call's stream: what is given back is reused only behind the call's kernels."""
    if workspace is None:
        if need == 0:
            return None, 0, None
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=f"cuda:{device}")
        else:
            if isinstance(stream, int):      # (an ExternalStream of 0 would be one of torch's own)
                stream = torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream(device)
            with torch.cuda.stream(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device=f"cuda:{device}")
    else:
        _array(workspace, "workspace", torch.uint8, device)
    return workspace.data_ptr(), workspace.numel(), workspace


def _count(x, what):
    """A number that the library takes in 32 bits, which ctypes would cut without a word."""
    if not 0 <= x < 1 << 32:
        raise ValueError(f"{what} must be from 0 to 2^32 - 1, not {x}")
    return x


def _stream(stream, device):
    if stream is None:       # the current stream's handle, without a Stream object around it
        return torch._C._cuda_getCurrentRawStream(device)
    return stream if isinstance(stream, int) else stream.cuda_stream


def ibp_attn_prompt_workspace(q_heads, head_dim, q_rows, k_rows, n_seqs):
    out = _u64(0)
    check(lib().ibp_attn_prompt_workspace(_count(q_heads, "q_heads"), _count(head_dim, "head_dim"), _count(q_rows, "q_rows"),
                                          _count(k_rows, "k_rows"), _count(n_seqs, "n_seqs"), out), "ibp_attn_prompt_workspace")
    return out.value


def ibp_attn_prompt(q, k, v, q_starts, k_starts, out, lse=None, causal=True, scale=None, workspace=None, stream=None):
    """Attention of packed sequences: q [rows][q_heads][dim] against k, v [rows][kv_heads][dim] into
    out (like q) and lse (float32 [q_heads][q rows], or None); starts are int32 on the GPU."""
    device = _device(q, "q")
    if q.dtype not in TYPES:
        raise TypeError(f"q must be bfloat16 or float16, not {q.dtype}")
    rq = _rows(q, "q", q.dtype, device)
    heads, dim = q.shape[1:]
    rk = _rows(k, "k", q.dtype, device, None, dim)
    kv_heads = k.shape[1]
    rv = _rows(v, "v", q.dtype, device, kv_heads, dim)
    ro = _rows(out, "out", q.dtype, device, heads, dim)
    n = _starts(q_starts, k_starts, device)
    lse_at = None if lse is None else _array(lse, "lse", torch.float32, device, (heads, q.shape[0]))
    a = _attn(q, kv_heads, dim, scale, causal)
    need = ibp_attn_prompt_workspace(heads, dim, q.shape[0], k.shape[0], n) if workspace is None else 0
    at, size, held = _space(workspace, need, device, stream)
    check(lib().ibp_attn_prompt(a, rq, rk, rv, q_starts.data_ptr(), k_starts.data_ptr(), n, ro, lse_at, at, size,
                                _stream(stream, device)), "ibp_attn_prompt")


def ibp_attn_key_weights_workspace(q_heads, kv_heads, k_rows, n_seqs=1):
    out = _u64(0)
    check(lib().ibp_attn_key_weights_workspace(_count(q_heads, "q_heads"), _count(kv_heads, "kv_heads"), _count(k_rows, "k_rows"),
                                               _count(n_seqs, "n_seqs"), out), "ibp_attn_key_weights_workspace")
    return out.value


def ibp_attn_key_weights(q, k, q_starts, k_starts, lse, weights, causal=True, scale=None, workspace=None, stream=None):
    """The attention weight that every key received, into weights (float32 [kv_heads][k rows]); lse as
    ibp_attn_prompt left it."""
    device = _device(q, "q")
    if q.dtype not in TYPES:
        raise TypeError(f"q must be bfloat16 or float16, not {q.dtype}")
    rq = _rows(q, "q", q.dtype, device)
    heads, dim = q.shape[1:]
    rk = _rows(k, "k", q.dtype, device, None, dim)
    kv_heads = k.shape[1]
    n = _starts(q_starts, k_starts, device)
    lse_at = _array(lse, "lse", torch.float32, device, (heads, q.shape[0]))
    weights_at = _array(weights, "weights", torch.float32, device, (kv_heads, k.shape[0]))
    a = _attn(q, kv_heads, dim, scale, causal)
    need = ibp_attn_key_weights_workspace(heads, kv_heads, k.shape[0], n) if workspace is None else 0
    at, size, held = _space(workspace, need, device, stream)
    check(lib().ibp_attn_key_weights(a, rq, rk, q_starts.data_ptr(), k_starts.data_ptr(), n, lse_at, weights_at, at, size,
                                     _stream(stream, device)), "ibp_attn_key_weights")


def ibp_attn_decode_workspace(n_seqs, q_heads, kv_heads, head_dim, max_len, weights):
    out = _u64(0)
    check(lib().ibp_attn_decode_workspace(_count(n_seqs, "n_seqs"), _count(q_heads, "q_heads"), _count(kv_heads, "kv_heads"),
                                          _count(head_dim, "head_dim"), _count(max_len, "max_len"), int(bool(weights)), out),
          "ibp_attn_decode_workspace")
    return out.value


def ibp_attn_decode(q, k, v, table, lens, max_len, out, lse=None, weights=None, scale=None, workspace=None, stream=None):
    """Attention of one new token per sequence (q [sequences][q_heads][dim]) over the pages that table
    (int32 [sequences][pages]) names in the pools k and v, lens (int32) slots of each, at most max_len;
    adds each slot's weight to weights (float32 [sequences][kv_heads][slots]) unless that is None."""
    device = _device(q, "q")
    if q.dtype not in TYPES:
        raise TypeError(f"q must be bfloat16 or float16, not {q.dtype}")
    rq = _rows(q, "q", q.dtype, device)
    n, heads, dim = q.shape
    pages = _pages(k, v, table, device)
    kv_heads = k.shape[1]
    if k.dtype != q.dtype or k.shape[3] != dim:
        raise TypeError(f"keys and values must be {q.dtype} of head_dim {dim}")
    if table.shape[0] != n:
        raise ValueError("table must have a row for every sequence")
    lens_at = _array(lens, "lens", torch.int32, device, (n,))
    ro = _rows(out, "out", q.dtype, device, heads, dim)
    lse_at = None if lse is None else _array(lse, "lse", torch.float32, device, (n, heads))
    weights_at, slots = None, 0
    if weights is not None:
        if weights.dim() != 3 or weights.shape[:2] != (n, kv_heads):
            raise ValueError("weights must be [sequences][kv_heads][slots]")
        weights_at, slots = _array(weights, "weights", torch.float32, device), weights.shape[2]
    a = _attn(q, kv_heads, dim, scale)
    need = 0
    if workspace is None:
        need = ibp_attn_decode_workspace(n, heads, kv_heads, dim, max_len, weights is not None)
    at, size, held = _space(workspace, need, device, stream)
    check(lib().ibp_attn_decode(a, rq, pages, lens_at, _count(max_len, "max_len"), ro, lse_at, weights_at, slots, at, size,
                                _stream(stream, device)), "ibp_attn_decode")


def ibp_kv_evict_workspace(n_seqs, kv_heads, max_len, budget):
    out = _u64(0)
    check(lib().ibp_kv_evict_workspace(_count(n_seqs, "n_seqs"), _count(kv_heads, "kv_heads"), _count(max_len, "max_len"),
                                       _count(budget, "budget"), out), "ibp_kv_evict_workspace")
    return out.value


def ibp_kv_evict(k, v, table, lens, max_len, budget, recent, next_positions, weights, positions, new_weights, new_positions,
                 new_lens, workspace=None, stream=None):
    """Keeps `budget` slots of every sequence and KV head: the `recent` newest positions and the heaviest
    weights. weights (float32) and positions (int32) are [sequences][kv_heads][slots]; the new ones, of at
    least the kept slots, and new_lens may be the same tensors."""
    device = _device(k, "keys")
    pages = _pages(k, v, table, device)
    n, kv_heads, dim = table.shape[0], k.shape[1], k.shape[3]
    lens_at = _array(lens, "lens", torch.int32, device, (n,))
    next_at = _array(next_positions, "next_positions", torch.int32, device, (n,))
    new_lens_at = _array(new_lens, "new_lens", torch.int32, device, (n,))
    if weights.dim() != 3 or weights.shape[:2] != (n, kv_heads) or positions.shape != weights.shape:
        raise ValueError("weights and positions must be [sequences][kv_heads][slots]")
    if new_weights.dim() != 3 or new_weights.shape[:2] != (n, kv_heads) or new_positions.shape != new_weights.shape:
        raise ValueError("new_weights and new_positions must be [sequences][kv_heads][slots]")
    weights_at = _array(weights, "weights", torch.float32, device)
    positions_at = _array(positions, "positions", torch.int32, device)
    new_weights_at = _array(new_weights, "new_weights", torch.float32, device)
    new_positions_at = _array(new_positions, "new_positions", torch.int32, device)
    a = ibp_attn(TYPES[k.dtype], kv_heads, kv_heads, dim, 1.0, 0)
    need = ibp_kv_evict_workspace(n, kv_heads, max_len, budget) if workspace is None else 0
    at, size, held = _space(workspace, need, device, stream)
    check(lib().ibp_kv_evict(a, pages, lens_at, n, _count(max_len, "max_len"), _count(budget, "budget"),
                             _count(recent, "recent"), next_at, weights_at, positions_at, weights.shape[2], new_weights_at,
                             new_positions_at, new_weights.shape[2], new_lens_at, at, size, _stream(stream, device)),
          "ibp_kv_evict")
