"""The attention operators' definitions in 64 bits on the CPU, and how far 32-bit sums of rounded
weights may be from them. Shares no code with the library.

Bounds, from the unit roundoffs u32 = 2^-24 (sums, products with exact inputs) and u (2^-8 for
bfloat16, 2^-11 for float16), worst case throughout:
  a score      (dim + 4) u32 scale sum |q_d k_d|: the products of 2-byte values are exact in 32 bits, their
               sum is not; then scale and the exponent's argument, 4 u32 |score| (scale sum |q k| bounds it)
  an exponential   its argument's error, and 2^-22 of its own
  a sum of n weights   n u32
  lse          the scores' error + n u32 + 2^-22 + 4 u32 |lse|, and u32-size errors of the reference m scale
  out          weights rounded to u: u sum p |v|; the exponentials' error and the sum's on both sides of the
               quotient; the output's own rounding u |out|; and in float16 the spacing 2^-24 below 2^-14, for
               weights (relative to a sum of at least 1) and the output
"""
import torch

U32 = 2.0 ** -24
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
NEG = float("-inf")


def visible(q_len, k_len, causal):
    i, j = torch.arange(q_len)[:, None], torch.arange(k_len)[None, :]
    return (j <= i + k_len - q_len) if causal else torch.ones(q_len, k_len, dtype=torch.bool)


def attend(q, k, v, scale, seen):
    """One head: q [n][d], k and v [m][d]. Returns out, lse and their bounds; what a row does not see is
    never read for it."""
    kind = q.dtype
    n, m, dim = q.shape[0], k.shape[0], q.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, lse = torch.zeros(n, v.shape[1], dtype=torch.float64), torch.full((n,), NEG, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    u = UNIT[kind]
    for i in range(n):
        at = seen[i].nonzero()[:, 0]
        if at.numel() == 0:
            continue
        x = (k[at] @ q[i]) * scale
        err = ((k[at].abs() @ q[i].abs()) * scale * (dim + 8) * U32).max()
        lse[i] = torch.logsumexp(x, 0)
        if lse[i] == NEG:
            continue
        p = (x - lse[i]).exp()
        out[i] = p @ v[at]
        weight = p @ v[at].abs()
        rel = err + 2.0 ** -22 + at.numel() * U32
        lse_tol[i] = rel + 8 * U32 * (lse[i].abs() + x.abs().max())
        out_tol[i] = 1.01 * (u * weight + u * out[i].abs() + 2 * rel * weight)
        if kind == torch.float16:
            out_tol[i] += 2.0 ** -24 * (v[at].abs().sum(0) + 1)
    return out, lse, out_tol, lse_tol


def key_weights(q, k, lse, scale, seen):
    """One query head's weights per key for given lse (float32), and their bound."""
    dim = q.shape[1]
    q, k, lse = q.double(), k.double(), lse.double()
    w, tol = torch.zeros(k.shape[0], dtype=torch.float64), torch.zeros(k.shape[0], dtype=torch.float64)
    for j in range(k.shape[0]):
        at = (seen[:, j] & (lse != NEG)).nonzero()[:, 0]
        if at.numel() == 0:
            continue
        x = (q[at] @ k[j]) * scale
        err = ((q[at].abs() @ k[j].abs()) * scale * (dim + 8) * U32).max() + 4 * U32 * lse[at].abs().max()
        w[j] = (x - lse[at]).exp().sum()
        tol[j] = 1.01 * w[j] * (err + 2.0 ** -22 + (at.numel() + 64) * U32)
    return w, tol


def evict(weights, positions, lens, next_positions, budget, recent):
    """Per (sequence, head): the slot whose content each of the first m slots has afterwards."""
    import math
    result = []
    weights, positions = weights.tolist(), positions.tolist()
    for b in range(len(weights)):
        heads = []
        for h in range(len(weights[b])):
            n = lens[b]
            m = min(n, budget)
            rank = []
            for i in range(n):
                w = weights[b][h][i]
                guarded = positions[b][h][i] >= next_positions[b] - recent
                rank.append((not guarded, 0.0 if guarded else -NEG if math.isnan(w) else -w, i))
            kept = sorted(i for _, _, i in sorted(rank)[:m])
            source = list(range(m))
            stay = set(kept)
            holes = [i for i in range(m) if i not in stay]
            for to, of in zip(holes, [i for i in kept if i >= m]):
                source[to] = of
            heads.append(source)
        result.append(heads)
    return result
