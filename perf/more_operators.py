"""The operators that write a paged KV cache and that hold it in 4 bits, as cases to be timed and compared.

What follows a layer's projections in serving: keys turned by their positions and appended to the
cache's pages, the queries turned with them (`append`); the same into a cache of 4 bits a value
(`append4`, read back as the next prompt's attention would); a 4-bit cache's rows as packed 16-bit
ones, for a prompt against its history (`read4`); and one new token per sequence over the 4-bit cache
(`decode4`). Shapes follow the benchmark's KV cache (8 KV heads of 128, up to 32,768 tokens) and
common variants of it.

    listed()            the cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) the tensors of a serving program
    run(state)          one pass: the plain form, or with `own` the library's operator
    exact(case, seed)   the definition in 64 bits
    work(case)          bytes and operations that the pass cannot do without

A record is what a 4-bit cache holds of one token of one head, in groups of 32 values (G of them):
16 G bytes of codes (byte i: value 2 i in its low half, 2 i + 1 in its high half), G steps, G
centres, both in the cache's 16-bit type, padded to 16 bytes. Value = centre + (code - 7.5) step.
"""
import math
import random

import numpy as np
import torch
from torch.nn.functional import pad

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
NEG = float("-inf")


def listed():
    return [
        # the next token of one conversation: latency
        {"name": "append_one", "op": "append", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, "turned": 128,
         "halves": True, "seqs": 1, "new": 1, "history": 1530, "gone": 0, "page": 16, "tracked": False},
        # a serving batch's next tokens, in caches that are held at a budget (weights and positions of the slots)
        {"name": "append_batch", "op": "append", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, "turned": 128,
         "halves": True, "seqs": 64, "new": 1, "history": 500, "gone": 1000, "page": 32, "tracked": True},
        # a packed batch of turns of very different lengths, half of every head turned, in pairs of neighbours
        {"name": "append_packed", "op": "append", "type": "f16", "heads": 16, "kv_heads": 16, "dim": 64, "turned": 32,
         "halves": False, "seqs": 11, "new": 2501, "history": 300, "gone": 0, "page": 24, "tracked": True},
        # one long prompt
        {"name": "append_prompt", "op": "append", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, "turned": 128,
         "halves": True, "seqs": 1, "new": 8192, "history": 0, "gone": 0, "page": 64, "tracked": False},
        # a serving batch's next tokens into 4-bit caches
        {"name": "append4_batch", "op": "append4", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, "turned": 128,
         "halves": True, "seqs": 64, "new": 1, "history": 500, "gone": 1000, "page": 32, "tracked": True},
        # one long prompt into a 4-bit cache
        {"name": "append4_prompt", "op": "append4", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128, "turned": 128,
         "halves": True, "seqs": 1, "new": 8192, "history": 0, "gone": 0, "page": 64, "tracked": False},
        # the histories of a few conversations, for the attention of their next turn
        {"name": "read4_turn", "op": "read4", "type": "f16", "kv_heads": 16, "dim": 80, "seqs": 5, "longest": 777, "page": 16},
        # the history of the benchmark's length
        {"name": "read4_long", "op": "read4", "type": "bf16", "kv_heads": 8, "dim": 128, "seqs": 1, "longest": 32768, "page": 64},
        # the next token of one conversation: latency
        {"name": "decode4_one", "op": "decode4", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 1, "longest": 1531, "page": 16, "weights": False},
        # one very long context: few rows, all the work along the cache
        {"name": "decode4_long", "op": "decode4", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 1, "longest": 131071, "page": 64, "weights": False},
        # wide heads that share one pair of keys and values, ranked for eviction
        {"name": "decode4_wide", "op": "decode4", "type": "f16", "heads": 8, "kv_heads": 1, "dim": 256,
         "seqs": 24, "longest": 6000, "page": 32, "weights": True},
        # a full serving batch over ragged contexts, ranked for eviction
        {"name": "decode4_batch", "op": "decode4", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 64, "longest": 8192, "page": 32, "weights": True},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["append", "append4", "read4", "decode4", "decode4"])
    dim = rng.choice([40, 64, 80, 96, 128, 128, 256])
    heads, kv_heads = rng.choice([(32, 8), (16, 16), (28, 4), (16, 1), (8, 2)])
    case = {"op": op, "type": rng.choice(["bf16", "f16"]), "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "page": rng.choice([16, 24, 32, 64, 128])}
    if op in ("append", "append4"):
        seqs = _log(rng, 1, 64)
        new = 1 if rng.random() < 0.5 else _log(rng, 2, min(8192, 8192 * 32 * 128 // (seqs * max(heads, 2 * kv_heads) * dim)))
        return {**case, "turned": rng.choice([dim, dim, dim // 16 * 8]), "halves": rng.random() < 0.6, "seqs": seqs, "new": new,
                "history": rng.choice([0, _log(rng, 1, min(2000, 60000 // seqs))]), "gone": rng.choice([0, _log(rng, 1, 100000)]),
                "tracked": rng.random() < 0.5}
    if op == "read4":
        del case["heads"]
        seqs = _log(rng, 1, 16)
        return {**case, "seqs": seqs, "longest": _log(rng, 16, min(32768, 32768 * 8 * 128 // (seqs * kv_heads * dim)))}
    seqs = _log(rng, 1, 64)
    longest = _log(rng, 64, min(131071, 524288 * 128 // (seqs * kv_heads * dim)))
    return {**case, "seqs": seqs, "longest": longest, "weights": rng.random() < 0.5}


# ---------------------------------------------------------------- inputs

def _spread(n, longest, seed, down_to_one=False):
    """n lengths up to the longest, out of order: in equal steps, or in equal steps of the logarithm."""
    if down_to_one:
        lengths = [round(longest ** (1 - i / max(n - 1, 1))) for i in range(n)]
    else:
        lengths = [longest * (i + 1) // n for i in range(n)]
    random.Random(seed).shuffle(lengths)
    return lengths


def _lengths(case):
    """For appends each sequence's new rows and what it holds already; else its length."""
    n = case["seqs"]
    if case["op"] in ("append", "append4"):
        new = [1] * n if case["new"] == 1 else _spread(n, case["new"], n, True)
        return new, _spread(n, case["history"], n + 1)
    return [max(1, x) for x in _spread(n, case["longest"], n)]


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEVICE)


def _starts(lengths):
    return _int32(np.cumsum([0] + list(lengths)))


def _values(g, rows, heads, dim, kind):
    return torch.randn(rows, heads, dim, generator=g, device=DEVICE).to(kind)


def _keys(g, rows, heads, dim, kind):
    """Keys with two outlier channels in every head, as in the benchmark's KV cache."""
    x = torch.randn(rows, heads, dim, generator=g, device=DEVICE).mul_(0.5)
    channel = torch.rand(heads, dim, generator=g, device=DEVICE).argsort(1)[:, :2]
    gain = torch.ones(heads, dim, device=DEVICE).scatter_(1, channel, 6.0)
    return (x * gain).to(kind)


def _rotation(positions, turned):
    """Cosine and sine of every position and pair, [positions][pairs][2]; the angles in 64 bits."""
    rate = 10000.0 ** (-torch.arange(0, turned, 2, dtype=torch.float64, device=DEVICE) / turned)
    angle = torch.arange(positions, dtype=torch.float64, device=DEVICE)[:, None] * rate
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def _record_bytes(dim):
    return -(-20 * -(-dim // 32) // 16) * 16


def _pool(rows, n_pages, page):
    """Rows [token][head][...] of whole pages as a pool [page][head][token][...]."""
    return rows.view(n_pages, page, *rows.shape[1:]).transpose(1, 2).contiguous()


def prepare(case, seed):
    g, kind, dim, kv_heads = _generator(seed), TYPES[case["type"]], case["dim"], case["kv_heads"]
    s = {"case": dict(case), "kind": kind, "scale": dim ** -0.5}
    seqs, page = case["seqs"], case["page"]
    if case["op"] in ("append", "append4"):
        new, held = _lengths(case)
        lens = [a + b for a, b in zip(new, held)]
    else:
        lens = _lengths(case)
    per_seq = -(-max(lens) // page)
    n_pages = seqs * per_seq
    s["table"] = torch.randperm(n_pages, generator=g, device=DEVICE).view(seqs, per_seq).to(torch.int32)
    s["lens"], s["longest"] = _int32(lens), max(lens)
    rows = [make(g, n_pages * page, kv_heads, dim, kind) for make in (_keys, _values)]
    if case["op"] == "append":
        s["keys"], s["values"] = (_pool(x, n_pages, page) for x in rows)
    else:
        s["keys"], s["values"] = (_pool(_records(x.float(), kind), n_pages, page) for x in rows)
    del rows
    if case["op"] in ("append", "append4"):
        total = sum(new)
        s["k"], s["v"] = _keys(g, total, kv_heads, dim, kind), _values(g, total, kv_heads, dim, kind)
        s["q"] = _values(g, total, case["heads"], dim, kind)
        s["q_out"] = torch.empty_like(s["q"])
        s["starts"] = None if case["new"] == 1 else _starts(new)
        s["first"] = _int32(held)
        s["next"] = s["lens"] + case["gone"]
        s["rotation"] = _rotation(max(lens) + case["gone"], case["turned"])
        s["weights"] = s["positions"] = None
        if case["tracked"]:
            s["weights"] = torch.rand(seqs, kv_heads, per_seq * page, generator=g, device=DEVICE)
            s["positions"] = torch.randint(0, 1 << 20, (seqs, kv_heads, per_seq * page), generator=g, device=DEVICE, dtype=torch.int32)
        if case["op"] == "append4":
            s["k_out"], s["v_out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    elif case["op"] == "read4":
        s["starts"], s["first"] = _starts(lens), None
        s["k_out"], s["v_out"] = (torch.empty(sum(lens), kv_heads, dim, dtype=kind, device=DEVICE) for _ in range(2))
    else:
        s["q"] = _values(g, seqs, case["heads"], dim, kind)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(seqs, case["heads"], device=DEVICE)
        s["weights"] = torch.rand(seqs, kv_heads, max(lens), generator=g, device=DEVICE) if case["weights"] else None
        s["workspace"] = None
        if own:                          # the buffer that a program keeps for the library's intermediate results
            import paper_2605_30728_amd as ibp
            need = ibp.ibp_attn_decode4_workspace(seqs, case["heads"], kv_heads, dim, max(lens), case["weights"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEVICE)
    return s


# ---------------------------------------------------------------- the plain form

def _records(x, kind):
    """Rows [...][dim] in 32 bits as records [...][bytes]."""
    fill = -x.shape[-1] % 32
    groups = lambda y: pad(x, (0, fill), value=y).unflatten(-1, (-1, 32))  # noqa: E731
    lo, hi = groups(math.inf).amin(-1), groups(-math.inf).amax(-1)
    centre = (lo * 0.5 + hi * 0.5).to(kind).float()
    step = (torch.maximum(hi - centre, centre - lo) * (2 / 15)).to(kind).float()
    inverse = torch.where(step >= 2.0 ** -126, 1 / step, torch.zeros_like(step))
    code = ((groups(0.0) - centre[..., None]) * inverse[..., None] + 7.5).round().clamp(0, 15)
    code = code.to(torch.uint8).flatten(-2)
    if fill:
        code[..., x.shape[-1]:] = 0
    parts = [code[..., 0::2] | code[..., 1::2] << 4, step.to(kind).view(torch.uint8), centre.to(kind).view(torch.uint8)]
    record = torch.cat(parts, -1)
    return pad(record, (0, _record_bytes(x.shape[-1]) - record.shape[-1]))


def _values_of(record, dim, kind):
    """What records stand for, [...][dim] in 32 bits."""
    n = -(-dim // 32)
    code = record[..., :16 * n]
    code = torch.stack([code & 15, code >> 4], -1).flatten(-2).float().unflatten(-1, (n, 32))
    step = record[..., 16 * n:18 * n].contiguous().view(kind).float()
    centre = record[..., 18 * n:20 * n].contiguous().view(kind).float()
    return ((code - 7.5) * step[..., None] + centre[..., None]).flatten(-2)[..., :dim]


def _turn(s, x, position):
    """Rows [row][head][dim], their first values turned by their positions, in 32 bits."""
    x, half = x.float(), s["case"]["turned"] // 2
    t = s["rotation"][position][:, None]
    cos, sin = t[..., 0], t[..., 1]
    out = x.clone()
    first, second = ((slice(0, half), slice(half, 2 * half)) if s["case"]["halves"] else
                     (slice(0, 2 * half, 2), slice(1, 2 * half, 2)))
    a, b = x[..., first], x[..., second]
    out[..., first] = a * cos - b * sin
    out[..., second] = a * sin + b * cos
    return out


def _rows_at(s, rows):
    """Sequence and place in it of every packed row."""
    row = torch.arange(rows, device=DEVICE)
    if s["starts"] is None:
        return row, torch.zeros_like(row)
    seq = torch.searchsorted(s["starts"][1:].long(), row, right=True)
    return seq, row - s["starts"][seq].long()


def _slots(s, seq, slot):
    """Page and row in it of slots."""
    page = s["case"]["page"]
    return s["table"].long()[seq, slot // page], slot % page


def _append(s):
    c, kind = s["case"], s["kind"]
    rows = s["k"].shape[0]
    seq, place = _rows_at(s, rows)
    back = (torch.ones_like(s["lens"]) if s["starts"] is None else s["starts"].diff()).long()[seq] - place
    slot, position = s["lens"].long()[seq] - back, s["next"].long()[seq] - back
    s["q_out"].copy_(_turn(s, s["q"], position))
    page, row = _slots(s, seq, slot)
    k, v = _turn(s, s["k"], position), s["v"]
    if c["op"] == "append4":
        k, v = _records(k, kind), _records(v.float(), kind)
    s["keys"][page, :, row], s["values"][page, :, row] = k.to(s["keys"].dtype), v
    out = {"q": s["q_out"]}
    if c["tracked"]:
        s["weights"][seq, :, slot] = 0.0
        s["positions"][seq, :, slot] = position[:, None].to(torch.int32).expand(-1, c["kv_heads"])
        out = {**out, "weights": s["weights"], "positions": s["positions"]}
    if c["op"] == "append":
        return {**out, "keys": s["keys"], "values": s["values"]}
    return {**out, **_read(s)}


def _read(s):
    seq, place = _rows_at(s, s["k_out"].shape[0])
    slot = place if s["first"] is None else place + s["first"].long()[seq]
    page, row = _slots(s, seq, slot)
    s["k_out"].copy_(_values_of(s["keys"][page, :, row], s["case"]["dim"], s["kind"]))
    s["v_out"].copy_(_values_of(s["values"][page, :, row], s["case"]["dim"], s["kind"]))
    return {"k": s["k_out"], "v": s["v_out"]}


def _decode(s):
    c = s["case"]
    k, v = (_values_of(pool[s["table"].long()].transpose(1, 2).flatten(2, 3), c["dim"], s["kind"]) for pool in (s["keys"], s["values"]))
    q = s["q"].float().unflatten(1, (c["kv_heads"], -1))
    live = torch.arange(k.shape[2], device=DEVICE) < s["lens"][:, None]
    x = (q @ k.transpose(-1, -2).contiguous()).mul_(s["scale"]).masked_fill_(~live[:, None, None], NEG)
    top = x.amax(-1, keepdim=True)
    p = (x - top).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(total)
    s["out"].copy_((p @ v).flatten(1, 2))
    s["lse"].copy_((top + total.log()).squeeze(-1).flatten(1, 2))
    out = {"out": s["out"], "lse": s["lse"]}
    if s["weights"] is not None:
        out["weights"] = s["weights"].add_(p.sum(2)[..., :s["longest"]])
    return out


# ---------------------------------------------------------------- the pass

def run(state):
    s, c = state, state["case"]
    if not own:
        return {"append": _append, "append4": _append, "read4": _read, "decode4": _decode}[c["op"]](s)
    import paper_2605_30728_amd as ibp
    if c["op"] == "decode4":
        ibp.ibp_attn_decode4(s["q"], s["keys"], s["values"], s["table"], s["lens"], s["longest"], s["out"], s["lse"],
                             weights=s["weights"], scale=s["scale"], workspace=s["workspace"])
        out = {"out": s["out"], "lse": s["lse"]}
        return out if s["weights"] is None else {**out, "weights": s["weights"]}
    out = {}
    if c["op"] != "read4":
        append = ibp.ibp_kv_append if c["op"] == "append" else ibp.ibp_kv4_append
        append(s["k"], s["v"], s["keys"], s["values"], s["table"], s["lens"], s["next"], starts=s["starts"],
               rotation=s["rotation"], halves=c["halves"], q=s["q"], q_out=s["q_out"], weights=s["weights"],
               positions=s["positions"])
        out = {"q": s["q_out"]}
        if c["tracked"]:
            out = {**out, "weights": s["weights"], "positions": s["positions"]}
        if c["op"] == "append":
            return {**out, "keys": s["keys"], "values": s["values"]}
    ibp.ibp_kv4_read(s["keys"], s["values"], s["table"], s["lens"], s["k_out"], s["v_out"], starts=s["starts"], first=s["first"])
    return {**out, "k": s["k_out"], "v": s["v_out"]}


# ---------------------------------------------------------------- the definition in 64 bits

def _stands_for(records, dim, kind):
    """Of records, [row][head][bytes], by looking each byte's two values up."""
    n = -(-dim // 32)
    byte = torch.arange(256, device=DEVICE)
    pairs = torch.stack([byte % 16, byte // 16], 1).double() - 7.5
    steps, centres = records[..., 16 * n:20 * n].contiguous().view(kind).double().split(n, -1)
    x = pairs[records[..., :16 * n].long()].reshape(*records.shape[:-1], n * 32)
    return (x * steps.repeat_interleave(32, -1) + centres.repeat_interleave(32, -1))[..., :dim]


def _held(x, kind):
    """What rows of 64 bits are held as in 4: group by group, the definition."""
    out = torch.empty_like(x)
    for d in range(0, x.shape[-1], 32):
        y = x[..., d:d + 32]
        lo, hi = y.aminmax(dim=-1, keepdim=True)
        centre = ((lo + hi) / 2).to(kind).double()
        step = (torch.maximum(hi - centre, centre - lo) / 7.5).to(kind).double()
        level = torch.where(step > 0, ((y - centre) / step + 7.5).round().clamp(0, 15), torch.full_like(y, 8.0))
        out[..., d:d + 32] = centre + (level - 7.5) * step
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c, kind, dim = s["case"], s["kind"], case["dim"]
    table, lens = s["table"].long(), s["lens"].tolist()
    if c["op"] == "read4":
        parts = []
        for pool in (s["keys"], s["values"]):
            rows = [pool[table[b, :-(-n // c["page"])]].transpose(1, 2).flatten(0, 1)[:n] for b, n in enumerate(lens)]
            parts.append(_stands_for(torch.cat(rows), dim, kind))
        return {"k": parts[0], "v": parts[1]}
    if c["op"] == "decode4":
        group = c["heads"] // c["kv_heads"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEVICE)
        weights = s["weights"].double() if c["weights"] else None
        for b, n in enumerate(lens):
            at = table[b, :-(-n // c["page"])]
            for g in range(c["kv_heads"]):
                k, v = (_stands_for(pool[at, g].reshape(-1, pool.shape[-1])[:n], dim, kind) for pool in (s["keys"], s["values"]))
                heads = slice(g * group, (g + 1) * group)
                x = (s["q"][b, heads].double() @ k.t().contiguous()) * s["scale"]
                lse[b, heads] = torch.logsumexp(x, -1)
                p = (x - lse[b, heads, None]).exp_()
                out[b, heads] = p @ v
                if weights is not None:
                    weights[b, g, :n] += p.sum(0)
        return {"out": out, "lse": lse} if weights is None else {"out": out, "lse": lse, "weights": weights}
    # appends, sequence by sequence: its last rows in their order, pairs turned as complex numbers
    new, held = _lengths(case)
    half = c["turned"] // 2
    q, k = s["q"].double(), s["k"].double()
    spin = torch.view_as_complex(s["rotation"].double())
    at = 0
    for b, n in enumerate(new):
        position = held[b] + c["gone"]
        z = spin[position:position + n, None]
        for x in (q[at:at + n], k[at:at + n]):
            y = x[..., :2 * half].unflatten(-1, (2, half) if c["halves"] else (half, 2))
            pairs = y.transpose(-1, -2).contiguous() if c["halves"] else y.contiguous()
            pairs = torch.view_as_real(torch.view_as_complex(pairs) * z)
            y.copy_(pairs.transpose(-1, -2) if c["halves"] else pairs)
        at += n
    out = {"q": q}
    if c["tracked"]:
        weights, positions = s["weights"].double(), s["positions"]
        for b, n in enumerate(new):
            weights[b, :, held[b]:held[b] + n] = 0
            positions[b, :, held[b]:held[b] + n] = torch.arange(n, device=DEVICE, dtype=torch.int32) + held[b] + c["gone"]
        out = {**out, "weights": weights, "positions": positions}
    if c["op"] == "append4":
        return {**out, "k": _held(k, kind), "v": _held(s["v"].double(), kind)}
    pools, at = [s["keys"].double(), s["values"].double()], 0
    for b, n in enumerate(new):
        slot = torch.arange(held[b], held[b] + n, device=DEVICE)
        for pool, rows in zip(pools, (k, s["v"].double())):
            pool[table[b, slot // c["page"]], :, slot % c["page"]] = rows[at:at + n]
        at += n
    return {**out, "keys": pools[0], "values": pools[1]}


def work(case):
    dim, kv_heads, lengths = case["dim"], case["kv_heads"], _lengths(case)
    record = 20 * -(-dim // 32)
    if case["op"] in ("append", "append4"):
        rows = sum(lengths[0])
        pages = sum(-(-(a + b) // case["page"]) - b // case["page"] for a, b in zip(*lengths))
        moved = 2 * 2 * dim * case["heads"] + (8 * dim if case["op"] == "append" else 4 * dim + 2 * record + 4 * dim) * kv_heads
        return {"bytes": rows * (moved + 4 * case["turned"] + (8 * kv_heads if case["tracked"] else 0)) + 4 * pages,
                "flops": rows * (3 * case["turned"] * (case["heads"] + kv_heads) + (0 if case["op"] == "append" else 16 * dim * kv_heads))}
    total = sum(lengths)
    pages = sum(-(-n // case["page"]) for n in lengths)
    if case["op"] == "read4":
        return {"bytes": total * kv_heads * (2 * record + 4 * dim) + 4 * pages, "flops": 4 * dim * kv_heads * total}
    heads = case["heads"]
    return {"bytes": 2 * record * kv_heads * total + 4 * dim * heads * len(lengths) + 4 * pages
            + (8 * kv_heads * total if case["weights"] else 0), "flops": 4 * dim * heads * total}
