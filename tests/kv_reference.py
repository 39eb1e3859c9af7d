"""The operators that write a paged KV cache and hold it in 4 bits, on the CPU: their definitions in 64 bits
with bounds, and where the definition is one of 32-bit operations, those. Shares no code with the library.

Bounds, from the unit roundoffs u32 = 2^-24 and u (2^-8 for bfloat16, 2^-11 for float16):
  a turned value   two products and a sum in 32 bits, 3 u32 (|x c| + |y s|), and its own rounding, u of itself
                   (float16: 2^-25 at least)
  a held value     half a step from what it holds: the nearest code's, or at the ends 15/2 of the step's own
                   rounding, which is less; and 32-bit errors of its argument, 8 u32 (|x| + |centre| + 8 step)
  decode           as in attention_reference.py, where a key (code - 15/2) step + centre is summed as (16 + code)
                   and 47/2 apart, so that 55 step + |centre| stands for |k| in the score's error, in dim + 24 sums; weights
                   are rounded with their slot's step: u sum p step 15/2, and n u32 sum p (55 step + |centre|). Weights
                   times steps are float16 numbers times at least 4 2^12 over the largest step: half its spacing is 2^-25,
                   so n 15/2 2^-39 of the largest step
"""
import torch

from attention_reference import NEG, U32, UNIT

GROUP = 32


def groups_of(dim):
    return -(-dim // GROUP)


def record_bytes(dim):
    return -(-20 * groups_of(dim) // 16) * 16


def rotation_table(positions, pairs, base=10000.0):
    rate = base ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))
    angle = torch.arange(positions, dtype=torch.float64)[:, None] * rate
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def pairs_of(turned, halves):
    half = turned // 2
    i = torch.arange(half)
    return (i, i + half) if halves else (2 * i, 2 * i + 1)


def turn(x, angles, halves, kind=torch.float64):
    """One row [heads][dim] turned by angles [pairs][2], in 64 bits, or by 32-bit operations one by one."""
    x = x.to(kind)
    out = x.clone()
    a, b = pairs_of(2 * angles.shape[0], halves)
    c, s = angles.to(kind).unbind(-1)
    out[:, a] = x[:, a] * c - x[:, b] * s
    out[:, b] = x[:, a] * s + x[:, b] * c
    return out


def turn_bound(x, angles, halves):
    """What turn() may be off by in 32 bits before the last rounding."""
    x = x.double().abs()
    off = torch.zeros_like(x)
    a, b = pairs_of(2 * angles.shape[0], halves)
    c, s = angles.double().abs().unbind(-1)
    off[:, a] = 3 * U32 * (x[:, a] * c + x[:, b] * s)
    off[:, b] = 3 * U32 * (x[:, a] * s + x[:, b] * c)
    return off


def records_of(x, kind):
    """Rows [...][dim] of 32 bits as records, by the definition's 32-bit operations; padding 0."""
    dim, n = x.shape[-1], groups_of(x.shape[-1])
    assert x.numel()
    out = torch.zeros(*x.shape[:-1], record_bytes(dim), dtype=torch.uint8)
    for g in range(n):
        y = x[..., g * GROUP:(g + 1) * GROUP]
        lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
        centre = (lo * 0.5 + hi * 0.5).to(kind)
        c = centre.float()
        step = (torch.maximum(hi - c, c - lo) * torch.tensor(2 / 15, dtype=torch.float32)).to(kind)
        s = step.float()
        inverse = torch.where(s >= 2.0 ** -126, 1 / s, torch.zeros_like(s))
        code = ((y - c) * inverse + 7.5).round().clamp(0, 15)
        bad = ~(y.isfinite().all(-1, keepdim=True) & c.isfinite() & s.isfinite())
        code = torch.where(bad, torch.zeros_like(code), code).to(torch.uint8)
        nan = torch.tensor(float("nan"), dtype=kind)
        centre, step = torch.where(bad, nan, centre), torch.where(bad, nan, step)
        full = torch.zeros(*x.shape[:-1], GROUP, dtype=torch.uint8)
        full[..., :y.shape[-1]] = code
        out[..., 16 * g:16 * g + 16] = full[..., 0::2] | full[..., 1::2] << 4
        out[..., 16 * n + 2 * g:16 * n + 2 * g + 2] = step.contiguous().view(torch.uint8)
        out[..., 18 * n + 2 * g:18 * n + 2 * g + 2] = centre.contiguous().view(torch.uint8)
    return out


def parts_of(records, dim, kind, want=torch.float64):
    """code - 15/2, step and centre of every value of records [...][bytes]."""
    n = groups_of(dim)
    code = records[..., :16 * n].long()
    code = torch.stack([code % 16, code // 16], -1).flatten(-2)[..., :dim].to(want) - 7.5
    meta = records[..., 16 * n:20 * n].contiguous().view(kind).to(want)
    wide = lambda m: m.repeat_interleave(GROUP, -1)[..., :dim]  # noqa: E731
    return code, wide(meta[..., :n]), wide(meta[..., n:])


def values_of(records, dim, kind, want=torch.float64):
    code, step, centre = parts_of(records, dim, kind, want)
    return code * step + centre


def held_bound(x, records, kind):
    """How far records may be from the values x that they hold."""
    _, step, centre = parts_of(records, x.shape[-1], kind)
    return step / 2 * 1.001 + 8 * U32 * (x.double().abs() + centre.abs() + 8 * step)


def attend4(q, keys, values, scale):
    """One query head [dim] over records [n][bytes] of both. Returns out, lse and their bounds."""
    kind, dim, n = q.dtype, q.shape[0], keys.shape[0]
    out, out_tol = torch.zeros(dim, dtype=torch.float64), torch.zeros(dim, dtype=torch.float64)
    if n == 0:
        return out, torch.tensor(NEG, dtype=torch.float64), out_tol, torch.zeros((), dtype=torch.float64)
    kc, ks, kz = parts_of(keys, dim, kind)
    vc, vs, vz = parts_of(values, dim, kind)
    q = q.double()
    x = ((kc * ks + kz) @ q) * scale
    err = (((55 * ks + kz.abs()) @ q.abs()) * scale * (dim + 24) * U32).max()
    lse = torch.logsumexp(x, 0)
    p = (x - lse).exp()
    out = p @ (vc * vs + vz)
    rel = err + 2.0 ** -22 + n * U32
    lse_tol = rel + 8 * U32 * (lse.abs() + x.abs().max())
    whole = p @ (7.5 * vs + vz.abs())
    out_tol = 1.01 * (UNIT[kind] * (p @ (7.5 * vs)) + UNIT[kind] * out.abs() + 2 * rel * whole + (n + 8) * U32 * (p @ (55 * vs + vz.abs())))
    out_tol += n * 7.5 * 2.0 ** -39 * vs.max()
    if kind == torch.float16:
        out_tol += 2.0 ** -24
    return out, lse, out_tol, lse_tol


def weights4(q, keys, scale):
    """What one query head adds to the slots' weights, and the bound."""
    kind, dim = q.dtype, q.shape[0]
    kc, ks, kz = parts_of(keys, dim, kind)
    x = ((kc * ks + kz) @ q.double()) * scale
    err = (((55 * ks + kz.abs()) @ q.double().abs()) * scale * (dim + 24) * U32).max()
    w = (x - torch.logsumexp(x, 0)).exp()
    return w, w * (2 * err + 2.0 ** -21 + (keys.shape[0] + 16) * U32 + 16 * U32 * x.abs().max())
