"""The attention operators over KV tensors, as cases to be timed and compared.

One KV cache through its life in serving: attention over whole prompts (`prompt`), the attention
weight that every key received from them (`key_weights`), one new token per sequence over the
paged cache (`decode`), and eviction of the lightest tokens (`evict`). Shapes follow the
benchmark's KV cache (8 KV heads of 128 bf16, up to 32,768 tokens) and common variants of it.

    listed()            the cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) the tensors of a serving program
    run(state)          one pass: the plain form, or with `own` the library's operator
    exact(case, seed)   the definition in 64 bits
    work(case)          bytes and operations that the pass cannot do without
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
NEG = float("-inf")


def listed():
    return [
        # one short prompt (a chat turn): latency
        {"name": "prompt_short", "op": "prompt", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 1, "longest": 77, "history": 0, "causal": True},
        # a packed batch of prompts of very different lengths, 1 token among them
        {"name": "prompt_packed", "op": "prompt", "type": "f16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 11, "longest": 2501, "history": 0, "causal": True},
        # a chunk of a prompt against everything before it, every head with its own keys
        {"name": "prompt_chunk", "op": "prompt", "type": "bf16", "heads": 16, "kv_heads": 16, "dim": 64,
         "seqs": 1, "longest": 1000, "history": 8001, "causal": True},
        # one long prompt
        {"name": "prompt_long", "op": "prompt", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 1, "longest": 8192, "history": 0, "causal": True},
        # what the packed prompts gave each key, to rank the cache by
        {"name": "weights_packed", "op": "key_weights", "type": "f16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 11, "longest": 2501, "history": 0, "causal": True},
        # the same after the long prompt
        {"name": "weights_long", "op": "key_weights", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 1, "longest": 8192, "history": 0, "causal": True},
        # the next token of one conversation: latency
        {"name": "decode_one", "op": "decode", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 1, "longest": 1531, "page": 16, "weights": False},
        # one very long context: few rows, all the work along the cache
        {"name": "decode_long", "op": "decode", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 1, "longest": 131071, "page": 64, "weights": False},
        # wide heads that share one pair of keys and values, ranked for eviction
        {"name": "decode_wide", "op": "decode", "type": "f16", "heads": 8, "kv_heads": 1, "dim": 256,
         "seqs": 24, "longest": 6000, "page": 32, "weights": True},
        # a full serving batch over ragged contexts, ranked for eviction
        {"name": "decode_batch", "op": "decode", "type": "bf16", "heads": 32, "kv_heads": 8, "dim": 128,
         "seqs": 64, "longest": 8192, "page": 32, "weights": True},
        # every step of a cache at its budget: one token too many per head
        {"name": "evict_step", "op": "evict", "type": "bf16", "kv_heads": 8, "dim": 128, "seqs": 16,
         "longest": 2049, "budget": 2048, "recent": 256, "page": 32, "scattered": True},
        # once after the prompts: 32,768 tokens down to an eighth
        {"name": "evict_prompt", "op": "evict", "type": "bf16", "kv_heads": 8, "dim": 128, "seqs": 4,
         "longest": 32768, "budget": 4096, "recent": 1024, "page": 32, "scattered": False},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["prompt", "key_weights", "decode", "decode", "evict"])
    dim = rng.choice([64, 80, 96, 128, 128, 256])
    heads, kv_heads = rng.choice([(32, 8), (16, 16), (28, 4), (16, 1), (8, 2)])
    case = {"op": op, "type": rng.choice(["bf16", "f16"]), "heads": heads, "kv_heads": kv_heads, "dim": dim}
    if op in ("prompt", "key_weights"):
        case = {**case, "seqs": _log(rng, 1, 16), "longest": _log(rng, 16, 8192),
                "history": rng.choice([0, 0, _log(rng, 1, 4000)]), "causal": rng.random() < 0.8}
        while (work(case)["flops"] > 5e11
               or case["seqs"] * heads * case["longest"] * (case["longest"] + case["history"]) > 2 ** 31):
            case["longest"] = case["longest"] * 4 // 5      # (the plain form holds every pair in 32 bits)
        return case
    if op == "decode":
        seqs = _log(rng, 1, 64)
        longest = _log(rng, 64, min(131071, 524288 * 128 // (seqs * kv_heads * dim)))
        return {**case, "seqs": seqs, "longest": longest, "page": rng.choice([16, 24, 32, 64, 128]),
                "weights": rng.random() < 0.5}
    del case["heads"]
    seqs = _log(rng, 1, 16)
    longest = _log(rng, 64, 16384)
    budget = longest - 1 if rng.random() < 0.4 else rng.randint(longest // 8, longest - 1)
    return {**case, "seqs": seqs, "longest": longest, "budget": budget, "recent": rng.randint(0, budget // 2),
            "page": rng.choice([16, 24, 32, 64, 128]), "scattered": rng.random() < 0.5}


# ---------------------------------------------------------------- inputs

def _lengths(case):
    """The sequences' lengths: for prompts from the longest down to one token, equal steps of
    the logarithm; for decoding spread evenly and out of order; for eviction all the same."""
    n, longest = case["seqs"], case["longest"]
    if n == 1 or case["op"] == "evict":
        return [longest] * n
    if case["op"] == "decode":
        lengths = [max(1, longest * (i + 1) // n) for i in range(n)]
    else:
        lengths = [round(longest ** (1 - i / (n - 1))) for i in range(n)]
    random.Random(n).shuffle(lengths)
    return lengths


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _starts(lengths):
    return torch.tensor(np.cumsum([0] + list(lengths)), dtype=torch.int32, device=DEVICE)


def _values(g, rows, heads, dim, kind):
    return torch.randn(rows, heads, dim, generator=g, device=DEVICE).to(kind)


def _keys(g, rows, heads, dim, kind):
    """Keys with two outlier channels in every head, as in the benchmark's KV cache."""
    x = torch.randn(rows, heads, dim, generator=g, device=DEVICE).mul_(0.5)
    channel = torch.rand(heads, dim, generator=g, device=DEVICE).argsort(1)[:, :2]
    gain = torch.ones(heads, dim, device=DEVICE).scatter_(1, channel, 6.0)
    return (x * gain).to(kind)


def prepare(case, seed):
    g, kind, dim, kv_heads = _generator(seed), TYPES[case["type"]], case["dim"], case["kv_heads"]
    lengths = _lengths(case)
    s = {"case": dict(case), "scale": dim ** -0.5}
    need = 0
    if own:                              # the buffer that a program keeps for the library's intermediate results
        import paper_2605_30728_amd as ibp
        if case["op"] == "key_weights":
            need = ibp.ibp_attn_key_weights_workspace(case["heads"], kv_heads, sum(lengths) + case["history"] * len(lengths))
        elif case["op"] == "decode":
            need = ibp.ibp_attn_decode_workspace(case["seqs"], case["heads"], kv_heads, dim, max(lengths), case["weights"])
        elif case["op"] == "evict":
            need = ibp.ibp_kv_evict_workspace(case["seqs"], kv_heads, max(lengths), case["budget"])
    s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEVICE)
    if case["op"] in ("prompt", "key_weights"):
        k_lengths = [n + case["history"] for n in lengths]
        rows_q, rows_k = sum(lengths), sum(k_lengths)
        s["q"] = _values(g, rows_q, case["heads"], dim, kind)
        s["k"] = _keys(g, rows_k, kv_heads, dim, kind)
        s["q_starts"], s["k_starts"] = _starts(lengths), _starts(k_lengths)
        s["longest"] = (max(lengths), max(k_lengths))
        if case["op"] == "prompt":
            s["v"] = _values(g, rows_k, kv_heads, dim, kind)
            s["out"] = torch.empty(rows_q, case["heads"], dim, dtype=kind, device=DEVICE)
            s["lse"] = torch.empty(case["heads"], rows_q, device=DEVICE)
        else:
            s["lse"] = _lse(s)
            s["weights"] = torch.empty(kv_heads, rows_k, device=DEVICE)
        return s

    page, seqs = case["page"], case["seqs"]
    per_seq = -(-max(lengths) // page)
    n_pages = seqs * per_seq
    s["k"] = _keys(g, n_pages * page, kv_heads, dim, kind).view(n_pages, page, kv_heads, dim).transpose(1, 2).contiguous()
    s["v"] = _values(g, n_pages * page, kv_heads, dim, kind).view(n_pages, kv_heads, page, dim)
    s["table"] = torch.randperm(n_pages, generator=g, device=DEVICE).view(seqs, per_seq).to(torch.int32)
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEVICE)
    s["longest"] = max(lengths)
    if case["op"] == "decode":
        s["q"] = _values(g, seqs, case["heads"], dim, kind)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(seqs, case["heads"], device=DEVICE)
        s["weights"] = torch.rand(seqs, kv_heads, max(lengths), generator=g, device=DEVICE) if case["weights"] else None
    else:
        n, budget = case["longest"], case["budget"]
        # accumulated weights: a heavy tail, and some tokens that nothing looked at
        w = torch.randn(seqs, kv_heads, n, generator=g, device=DEVICE).mul_(2).exp_()
        s["weights"] = w * (torch.rand(seqs, kv_heads, n, generator=g, device=DEVICE) >= 0.05)
        order = torch.arange(n, device=DEVICE).expand(seqs, kv_heads, n)
        if case["scattered"]:
            order = torch.rand(seqs, kv_heads, n, generator=g, device=DEVICE).argsort(-1)
        s["positions"] = order.to(torch.int32).contiguous()
        s["next"] = s["lengths"].clone()
        s["new_weights"] = torch.zeros(seqs, kv_heads, budget, device=DEVICE)
        s["new_positions"] = torch.zeros(seqs, kv_heads, budget, dtype=torch.int32, device=DEVICE)
        s["new_lengths"] = torch.zeros_like(s["lengths"])
    return s


# ---------------------------------------------------------------- the plain form

def _padded(x, starts, longest):
    """The rows of packed sequences as [sequence][head][place][dim], in 32 bits."""
    at = starts[:-1, None].long() + torch.arange(longest, device=DEVICE)
    return x[at.clamp_(max=x.shape[0] - 1)].float().permute(0, 2, 1, 3)


def _places(starts, rows):
    """Sequence and place in it of every packed row."""
    row = torch.arange(rows, device=DEVICE)
    seq = torch.searchsorted(starts[1:].long(), row, right=True)
    return seq, row - starts[seq].long()


def _visible(s):
    """[sequence][1][query place][key place]: which keys a query sees."""
    q_len, k_len = s["q_starts"].diff().long(), s["k_starts"].diff().long()
    i = torch.arange(s["longest"][0], device=DEVICE)[:, None]
    j = torch.arange(s["longest"][1], device=DEVICE)[None, :]
    seen = (i < q_len[:, None, None]) & (j < k_len[:, None, None])
    if s["case"]["causal"]:
        seen &= j <= i + (k_len - q_len)[:, None, None]
    return seen[:, None]


def _scores(s):
    q = _padded(s["q"], s["q_starts"], s["longest"][0])
    k = _padded(s["k"], s["k_starts"], s["longest"][1])
    k = k.repeat_interleave(s["case"]["heads"] // s["case"]["kv_heads"], 1)
    return (q @ k.transpose(-1, -2).contiguous()).mul_(s["scale"]).masked_fill_(~_visible(s), NEG)


def _softmax(scores):
    """Weights (all zero where nothing is visible) and the logarithm of their denominators."""
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == NEG, torch.zeros_like(top), top)
    p = (scores - top).exp_()
    total = p.sum(-1, keepdim=True)
    p.mul_(torch.where(total == 0, total, 1 / total))
    return p, (top + total.log()).squeeze(-1)


def _packed(x, starts, rows):
    """[sequence][head][place]... back to packed rows, [row][head]..."""
    seq, place = _places(starts, rows)
    return x.transpose(1, 2)[seq, place]


def _lse(s):
    return _packed(_softmax(_scores(s))[1], s["q_starts"], s["q"].shape[0]).t().contiguous()


def _prompt(s):
    p, lse = _softmax(_scores(s))
    v = _padded(s["v"], s["k_starts"], s["longest"][1])
    out = p @ v.repeat_interleave(s["case"]["heads"] // s["case"]["kv_heads"], 1)
    rows = s["q"].shape[0]
    return {"out": _packed(out, s["q_starts"], rows).to(s["q"].dtype),
            "lse": _packed(lse, s["q_starts"], rows).t().contiguous()}


def _key_weights(s):
    seen = s["longest"][0]
    at = (s["q_starts"][:-1, None].long() + torch.arange(seen, device=DEVICE)).clamp_(max=s["q"].shape[0] - 1)
    lse = s["lse"][:, at].transpose(0, 1)[..., None]
    p = (_scores(s) - torch.where(lse == NEG, torch.zeros_like(lse), lse)).exp_()
    w = p.sum(-2).unflatten(1, (s["case"]["kv_heads"], -1)).sum(2)
    return {"weights": _packed(w, s["k_starts"], s["k"].shape[0]).t().contiguous()}


def _pages(pool, table):
    """[sequence][head][slot][dim] in 32 bits."""
    return pool[table.long()].transpose(1, 2).flatten(2, 3).float()


def _decode(s):
    c = s["case"]
    k, v = _pages(s["k"], s["table"]), _pages(s["v"], s["table"])
    q = s["q"].float().unflatten(1, (c["kv_heads"], -1))
    live = torch.arange(k.shape[2], device=DEVICE) < s["lengths"][:, None]
    scores = (q @ k.transpose(-1, -2).contiguous()).mul_(s["scale"]).masked_fill_(~live[:, None, None], NEG)
    p, lse = _softmax(scores)
    out = {"out": (p @ v).flatten(1, 2).to(s["q"].dtype), "lse": lse.flatten(1, 2)}
    if s["weights"] is not None:
        out["weights"] = s["weights"].add_(p.sum(2)[..., :s["longest"]])
    return out


def _rows_of(s, slot):
    """Rows of the pools, seen as [page][head][slot in page] rows, of [sequence][head][slot]."""
    c = s["case"]
    page = s["table"].long()[:, None].expand(-1, c["kv_heads"], -1).gather(2, slot // c["page"])
    head = torch.arange(c["kv_heads"], device=DEVICE)[:, None]
    return (page * c["kv_heads"] + head) * c["page"] + slot % c["page"]


def _evict(s):
    c = s["case"]
    n, budget = s["weights"].shape[-1], c["budget"]
    slot = torch.arange(n, device=DEVICE).expand(s["weights"].shape)
    live = slot < s["lengths"][:, None, None]
    guarded = s["positions"] >= (s["next"] - c["recent"])[:, None, None]
    w = s["weights"].nan_to_num(nan=NEG, posinf=float("inf"), neginf=NEG)
    order = w.argsort(dim=-1, descending=True, stable=True)
    first = (live.int() * 2 + (live & guarded).int()).gather(-1, order)
    order = order.gather(-1, first.argsort(dim=-1, descending=True, stable=True))
    rank = torch.empty_like(order).scatter_(-1, order, slot)
    keep = (rank < budget) & live
    kept = s["lengths"].clamp(max=budget).long()
    above = slot >= kept[:, None, None]
    hole, mover = ~keep & ~above, keep & above
    place = torch.where(mover, mover.long().cumsum(-1) - 1, torch.full_like(slot, n))
    by_rank = torch.zeros(*slot.shape[:-1], n + 1, dtype=torch.int64, device=DEVICE).scatter_(-1, place, slot)
    source = torch.where(hole, by_rank.gather(-1, (hole.long().cumsum(-1) - 1).clamp_(min=0)), slot)[..., :budget]
    to, of = _rows_of(s, slot[..., :budget]).flatten(), _rows_of(s, source).flatten()
    for pool in (s["k"], s["v"]):
        rows = pool.view(-1, pool.shape[-1])
        rows[to] = rows[of]
    s["new_weights"].copy_(s["weights"].gather(-1, source))
    s["new_positions"].copy_(s["positions"].gather(-1, source))
    s["new_lengths"].copy_(kept)
    return _evicted(s)


def _evicted(s):
    return {"weights": s["new_weights"], "positions": s["new_positions"], "lengths": s["new_lengths"], "k": s["k"], "v": s["v"]}


# ---------------------------------------------------------------- the pass

def run(state):
    s, c = state, state["case"]
    if not own:
        return {"prompt": _prompt, "key_weights": _key_weights, "decode": _decode, "evict": _evict}[c["op"]](s)
    import paper_2605_30728_amd as ibp
    if c["op"] == "prompt":
        ibp.ibp_attn_prompt(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"], s["out"], s["lse"],
                            causal=c["causal"], scale=s["scale"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "key_weights":
        ibp.ibp_attn_key_weights(s["q"], s["k"], s["q_starts"], s["k_starts"], s["lse"], s["weights"],
                                 causal=c["causal"], scale=s["scale"], workspace=s["workspace"])
        return {"weights": s["weights"]}
    if c["op"] == "decode":
        ibp.ibp_attn_decode(s["q"], s["k"], s["v"], s["table"], s["lengths"], s["longest"], s["out"], s["lse"],
                            weights=s["weights"], scale=s["scale"], workspace=s["workspace"])
        out = {"out": s["out"], "lse": s["lse"]}
        return out if s["weights"] is None else {**out, "weights": s["weights"]}
    ibp.ibp_kv_evict(s["k"], s["v"], s["table"], s["lengths"], s["longest"], c["budget"], c["recent"], s["next"],
                     s["weights"], s["positions"], s["new_weights"], s["new_positions"], s["new_lengths"],
                     workspace=s["workspace"])
    return _evicted(s)


# ---------------------------------------------------------------- the definition in 64 bits

def _attend(q, k, scale, offset):
    """Of one head: scores in 64 bits, key j seen by query i where j <= i + offset (None: all)."""
    x = (q.double() @ k.double().t().contiguous()).mul_(scale)
    if offset is not None:
        i, j = torch.arange(q.shape[0], device=DEVICE), torch.arange(k.shape[0], device=DEVICE)
        x.masked_fill_(j[None, :] > i[:, None] + offset, NEG)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    c, group = s["case"], case.get("heads", 0) // case["kv_heads"]
    if c["op"] in ("prompt", "key_weights"):
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        lse = torch.full((c["heads"], s["q"].shape[0]), NEG, dtype=torch.float64, device=DEVICE)
        weights = torch.zeros(c["kv_heads"], s["k"].shape[0], dtype=torch.float64, device=DEVICE)
        qs, ks = s["q_starts"].tolist(), s["k_starts"].tolist()
        for b in range(c["seqs"]):
            rq, rk = slice(qs[b], qs[b + 1]), slice(ks[b], ks[b + 1])
            offset = (rk.stop - rk.start) - (rq.stop - rq.start) if c["causal"] else None
            for h in range(c["heads"]):
                x = _attend(s["q"][rq, h], s["k"][rk, h // group], s["scale"], offset)
                if c["op"] == "prompt":
                    lse[h, rq] = torch.logsumexp(x, -1)
                    out[rq, h] = (x - lse[h, rq, None]).exp_() @ s["v"][rk, h // group].double()
                else:
                    weights[h // group, rk] += (x - s["lse"][h, rq, None].double()).exp_().sum(0)
        return {"out": out, "lse": lse} if c["op"] == "prompt" else {"weights": weights}
    table, lengths = s["table"].long(), s["lengths"].tolist()
    if c["op"] == "decode":
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEVICE)
        weights = s["weights"].double() if c["weights"] else None
        for b, n in enumerate(lengths):
            at = table[b, :-(-n // c["page"])]
            for g in range(c["kv_heads"]):
                k, v = (pool[at, g].reshape(-1, c["dim"])[:n] for pool in (s["k"], s["v"]))
                heads = slice(g * group, (g + 1) * group)
                x = _attend(s["q"][b, heads], k, s["scale"], None)
                lse[b, heads] = torch.logsumexp(x, -1)
                p = (x - lse[b, heads, None]).exp_()
                out[b, heads] = p @ v.double()
                if weights is not None:
                    weights[b, g, :n] += p.sum(0)
        return {"out": out, "lse": lse} if weights is None else {"out": out, "lse": lse, "weights": weights}
    new_w, new_p = s["new_weights"].double().cpu().numpy(), s["new_positions"].cpu().numpy()
    w, position = s["weights"].double().cpu().numpy(), s["positions"].cpu().numpy()
    table, k, v = table.cpu().numpy(), s["k"].clone(), s["v"].clone()
    for b, n in enumerate(lengths):
        m = min(n, c["budget"])
        for g in range(c["kv_heads"]):
            guarded = position[b, g, :n] >= n - c["recent"]
            kept = np.sort(np.lexsort((np.arange(n), -w[b, g, :n], ~guarded))[:m])
            source = np.arange(m)
            source[np.setdiff1d(source, kept)] = kept[kept >= m]
            new_w[b, g, :m], new_p[b, g, :m] = w[b, g, source], position[b, g, source]
            to, of = (np.divmod(x, c["page"]) for x in (np.arange(m), source))
            to, of = ((torch.from_numpy(table[b, x[0]]).to(DEVICE), torch.from_numpy(x[1]).to(DEVICE)) for x in (to, of))
            k[to[0], g, to[1]], v[to[0], g, to[1]] = s["k"][of[0], g, of[1]], s["v"][of[0], g, of[1]]
    device = lambda x: torch.from_numpy(x).to(DEVICE)  # noqa: E731
    return {"weights": device(new_w), "positions": device(new_p),
            "lengths": torch.tensor([min(n, c["budget"]) for n in lengths], dtype=torch.int32, device=DEVICE),
            "k": k.double(), "v": v.double()}


def work(case):
    lengths, dim, kv_heads = _lengths(case), case["dim"], case["kv_heads"]
    if case["op"] in ("prompt", "key_weights"):
        heads, past = case["heads"], case["history"]
        rows_q, rows_k = sum(lengths), sum(lengths) + past * len(lengths)
        pairs = sum(n * past + (n * (n + 1) // 2 if case["causal"] else n * n) for n in lengths)
        if case["op"] == "prompt":
            return {"bytes": 4 * dim * (heads * rows_q + kv_heads * rows_k) + 4 * heads * rows_q,
                    "flops": 4 * dim * heads * pairs}
        return {"bytes": 2 * dim * (heads * rows_q + kv_heads * rows_k) + 4 * heads * rows_q + 4 * kv_heads * rows_k,
                "flops": 2 * dim * heads * pairs}
    if case["op"] == "decode":
        heads, total = case["heads"], sum(lengths)
        pages = sum(-(-n // case["page"]) for n in lengths)
        return {"bytes": 4 * dim * (kv_heads * total + heads * len(lengths)) + 4 * pages
                + (8 * kv_heads * total if case["weights"] else 0), "flops": 4 * dim * heads * total}
    # expected moves: of the budget's slots, those that hold none of the kept tokens
    n, budget, recent = case["longest"], case["budget"], case["recent"]
    if case["scattered"]:
        moves = budget * (n - budget) / n
    else:
        old = n - recent
        moves = min(budget, old) * (1 - (budget - recent) / old) if old else 0
    per_head = 8 * n + 8 * budget + moves * 2 * 2 * 2 * dim
    return {"bytes": int(len(lengths) * kv_heads * per_head), "flops": len(lengths) * kv_heads * n}
