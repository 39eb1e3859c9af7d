"""One attention layer of a serving loop over a KV cache that was stored compressed.

Several conversations go on: their earlier keys and values lie in one compressed stream (a row is
one token of one head), a new turn of prompts comes in, then tokens one at a time, and the cache of
every conversation is held at a budget of slots.

    python examples/kv_serving.py

  1. restore   ibp_gather_decompress_device writes the stored rows straight into the cache's pages
               (row ids in the order of the pages), and once more packed for the prompts
  2. prompt    ibp_attn_prompt: the new turn's rows against history and turn, all sequences at once
  3. weights   ibp_attn_key_weights: what every key received from the turn
  4. append    ibp_kv_append: the turn's keys and values join the history in the pages
  5. evict     ibp_kv_evict: the most recent and the heaviest slots stay
  6. tokens    ibp_kv_append, ibp_attn_decode over the pages, which goes on adding up weights, then
               ibp_kv_evict in place

Queries, keys and values are random here; in a model they are the layer's projections, and ibp_kv_append turns them by
their positions on the way. With pools of ibp_kv4_record(dim) bytes a token, ibp_kv4_append, ibp_attn_decode4 and
ibp_kv4_read hold such a cache in 4 bits.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2605_30728_amd as ibp  # noqa: E402


def rows_of(history, kv_heads, dim, seed):
    """The conversations' earlier keys and values, [2][kv_heads][tokens of all][dim]."""
    g = np.random.default_rng(seed)
    tokens = sum(history)
    base = g.standard_normal((2, kv_heads, 1, dim))          # what the tokens of a head have in common
    return torch.from_numpy(base + 0.05 * g.standard_normal((2, kv_heads, tokens, dim))).bfloat16()


def store(rows):
    """Compresses them: a row of the stream is one token of one head."""
    return ibp.ibp_compress(rows.view(torch.int16).numpy().reshape(-1, rows.shape[-1]), 64)


class Cache:
    """A layer's paged KV cache: pools, page table, and per (sequence, head) the slots' weights and positions."""

    def __init__(self, seqs, kv_heads, dim, page, slots, device):
        self.page, self.slots = page, slots
        per = -(-slots // page)
        self.table = torch.arange(seqs * per, dtype=torch.int32, device=device).view(seqs, per)
        self.k = torch.zeros(seqs * per, kv_heads, page, dim, dtype=torch.bfloat16, device=device)
        self.v = torch.zeros_like(self.k)
        self.weights = torch.zeros(seqs, kv_heads, slots, device=device)
        self.positions = torch.zeros(seqs, kv_heads, slots, dtype=torch.int32, device=device)
        self.lens = torch.zeros(seqs, dtype=torch.int32, device=device)
        self.next = torch.zeros(seqs, dtype=torch.int32, device=device)

    def append(self, k, v, n=None):
        """The packed rows k, v [rows][kv_heads][dim], n (their numbers) of each sequence; None: one token of each."""
        starts = None
        if n is not None:
            starts = torch.tensor(np.concatenate(([0], np.cumsum(n))), dtype=torch.int32, device=self.k.device)
        more = 1 if n is None else starts.diff()
        self.lens += more
        self.next += more
        ibp.ibp_kv_append(k, v, self.k, self.v, self.table, self.lens, self.next, starts, weights=self.weights, positions=self.positions)

    def evict(self, budget, recent, longest):
        ibp.ibp_kv_evict(self.k, self.v, self.table, self.lens, longest, budget, recent, self.next, self.weights,
                         self.positions, self.weights, self.positions, self.lens)


def run(history=(700, 0, 1333), turn=(90, 33, 257), tokens=8, q_heads=32, kv_heads=8, dim=128, budget=512, recent=64,
        page=32, seed=0, on_token=None):
    """on_token(q, cache, out, weights before) is called after every token's attention."""
    device = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device="cpu").manual_seed(seed)
    random = lambda *shape: torch.randn(*shape, generator=g).to(device, torch.bfloat16)  # noqa: E731
    seqs, total, longest = len(history), sum(history), max(h + t for h, t in zip(history, turn))
    cache = Cache(seqs, kv_heads, dim, page, max(longest, budget + 1), device)
    k_starts = np.concatenate(([0], np.cumsum([h + t for h, t in zip(history, turn)]))).astype(np.int32)
    q_starts = np.concatenate(([0], np.cumsum(turn))).astype(np.int32)
    packed = torch.empty(2, int(k_starts[-1]), kv_heads, dim, dtype=torch.bfloat16, device=device)
    packed.copy_(random(*packed.shape))                      # the turn's rows; the history's follow
    new = packed.clone()

    # 1. stored row (x, head, token) is row (x * kv_heads + head) * total + token of the stream
    stream = store(rows_of(history, kv_heads, dim, seed)) if total else None
    handle = ibp.ibp_open(stream) if total else None
    heads = torch.arange(kv_heads, device=device)
    start = 0
    for b, h in enumerate(history):
        if h == 0:
            continue
        whole = -(-h // page) * page                         # to the page's end: the last token again, as padding
        token = torch.arange(whole, device=device).clamp(max=h - 1) + start
        for x, pool in enumerate((cache.k, cache.v)):
            ids = (x * kv_heads + heads[None, :, None]) * total + token.view(-1, 1, page)          # [page][head][row]
            first = int(cache.table[b, 0])                   # (this sequence's pages follow one another)
            ibp.ibp_gather_decompress_device(handle, ids.reshape(-1).contiguous(), pool[first:first + whole // page])
            ids = (x * kv_heads + heads[None, :]) * total + token[:h, None]                        # [token][head]
            ibp.ibp_gather_decompress_device(handle, ids.reshape(-1).contiguous(), packed[x, k_starts[b]:k_starts[b] + h])
        cache.positions[b, :, :h] = torch.arange(h, device=device, dtype=torch.int32)
        start += h
    cache.lens += torch.tensor(history, dtype=torch.int32, device=device)
    cache.next += cache.lens

    # 2. and 3. the new turn
    q = random(int(q_starts[-1]), q_heads, dim)
    starts = torch.from_numpy(q_starts).to(device), torch.from_numpy(k_starts).to(device)
    out = torch.empty_like(q)
    lse = torch.empty(q_heads, q.shape[0], device=device)
    weights = torch.zeros(kv_heads, packed.shape[1], device=device)
    ibp.ibp_attn_prompt(q, packed[0], packed[1], *starts, out, lse)
    ibp.ibp_attn_key_weights(q, packed[0], *starts, lse, weights)

    # 4.
    kept = [torch.arange(int(k_starts[b]) + h, int(k_starts[b + 1]), device=device) for b, h in enumerate(history)]
    cache.append(*new[:, torch.cat(kept)], turn)
    for b, (h, t) in enumerate(zip(history, turn)):
        n, at = h + t, int(k_starts[b])
        cache.weights[b, :, :n] = weights[:, at:at + n]
    prompt = dict(q=q, k=packed[0], v=packed[1], q_starts=q_starts, k_starts=k_starts, out=out, lse=lse, weights=weights)

    # 5.
    cache.evict(budget, recent, longest)

    # 6.
    held = min(longest, budget) + 1
    token_out = torch.empty(seqs, q_heads, dim, dtype=torch.bfloat16, device=device)
    workspace = torch.empty(max(ibp.ibp_attn_decode_workspace(seqs, q_heads, kv_heads, dim, cache.slots, True), 1),
                            dtype=torch.uint8, device=device)
    for _ in range(tokens):
        cache.append(random(seqs, kv_heads, dim), random(seqs, kv_heads, dim))
        q1 = random(seqs, q_heads, dim)
        before = cache.weights.clone() if on_token else None
        ibp.ibp_attn_decode(q1, cache.k, cache.v, cache.table, cache.lens, held, token_out, weights=cache.weights,
                            workspace=workspace)
        if on_token:
            on_token(q1, cache, token_out, before)
        cache.evict(budget, recent, held)
        held = min(held, budget) + 1
    torch.cuda.synchronize()
    if handle is not None:
        ibp.ibp_close(handle)
    return prompt, cache, None if stream is None else (len(stream), 4 * total * kv_heads * dim)


def main():
    if not torch.cuda.is_available():
        raise SystemExit("this example needs a GPU")
    prompt, cache, size = run()
    print(f"restored {size[1] / 1e6:.1f} MB of keys and values from {size[0] / 1e6:.1f} MB")
    print(f"prompt: {prompt['q'].shape[0]} rows against {prompt['k'].shape[0]} keys, then a token at a time")
    for b in range(len(cache.lens)):
        kept = cache.positions[b, 0, :cache.lens[b]].sort().values.tolist()
        print(f"sequence {b}: {int(cache.next[b])} tokens seen, {len(kept)} kept; head 0 keeps {kept[0]} .. {kept[-1]}, "
              f"total weight {float(cache.weights[b, :, :len(kept)].sum()):.1f}")


if __name__ == "__main__":
    main()
