"""Attention of single tokens over a paged cache, and eviction from it, against their definitions."""
import pytest
import torch

from attention_reference import UNIT, attend, evict

pytestmark = pytest.mark.gpu
NEG = float("-inf")
NAN = float("nan")
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ibp():
    import paper_2605_30728_amd
    return paper_2605_30728_amd


class Cache:
    """A paged cache on the CPU, its pages in no order, and everything outside the lengths NaN."""

    def __init__(self, kind, kv_heads, dim, lens, page, seed=0, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.kv_heads, self.dim = list(lens), page, kv_heads, dim
        self.per = max(-(-max(lens) // page), 1)
        n = len(lens) * self.per + spare
        self.k = torch.full((n, kv_heads, page, dim), NAN, dtype=kind)
        self.v = torch.full((n, kv_heads, page, dim), NAN, dtype=kind)
        self.table = torch.randperm(n, generator=g)[:len(lens) * self.per].view(len(lens), self.per).to(torch.int32)
        for b, length in enumerate(lens):
            for i in range(length):
                at = self.table[b, i // page].item(), slice(None), i % page
                self.k[at] = torch.randn(kv_heads, dim, generator=g).to(kind)
                self.v[at] = torch.randn(kv_heads, dim, generator=g).to(kind)

    def rows(self, pool, b, h, slots):
        slots = torch.as_tensor(slots, dtype=torch.long)
        return pool[self.table[b].long()[slots // self.page], h, slots % self.page]


def decode(ibp, c, q, weights=None, max_len=None, k=None, v=None, scale=None, lens=None, table=None):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    w = None if weights is None else weights.cuda()
    ibp.ibp_attn_decode(q.cuda(), c.k.cuda() if k is None else k, c.v.cuda() if v is None else v,
                        (c.table if table is None else table).cuda(),
                        torch.tensor(c.lens if lens is None else lens, dtype=torch.int32, device="cuda"),
                        max(c.lens) if max_len is None else max_len, out, lse, weights=w, scale=scale)
    return out.cpu(), lse.cpu(), None if w is None else w.cpu()


def check_decode(c, q, out, lse, before=None, after=None, slots=None):
    group = q.shape[1] // c.kv_heads
    scale = c.dim ** -0.5
    for b in range(q.shape[0]):
        at = list(range(c.lens[b])) if slots is None else slots[b]
        for g in range(c.kv_heads):
            k, v = c.rows(c.k, b, g, at), c.rows(c.v, b, g, at)
            added = torch.zeros(len(at), dtype=torch.float64)
            rel = 0.0
            for h in range(g * group, (g + 1) * group):
                o, x, o_tol, x_tol = attend(q[b, h:h + 1], k, v, scale, torch.ones(1, len(at), dtype=torch.bool))
                assert (lse[b, h] == NEG) == (x[0] == NEG)
                assert x[0] == NEG or abs(lse[b, h].double() - x[0]) <= x_tol[0]
                off = (out[b, h].double() - o[0]).abs()
                assert (off <= o_tol[0]).all(), (b, h, (off / o_tol[0].clamp(min=1e-30)).max())
                if at and before is not None:
                    added += ((k.double() @ q[b, h].double()) * scale - x[0]).exp()
                    rel = max(rel, 2 * x_tol[0].item())      # the score's error and the lse's
            if before is not None:
                want = before[b, g, at].double() + added
                assert ((after[b, g, at].double() - want).abs() <= added * (rel + (group + 4) * 2.0 ** -24) + want * 2.0 ** -23).all()
                rest = torch.ones(before.shape[2], dtype=torch.bool)
                rest[at] = False
                assert torch.equal(after[b, g, rest], before[b, g, rest])


def check_decode_head(c, q, out, lse):
    """The first query head of the sequences that are there."""
    for b in range(out.shape[0]):
        k, v = (c.rows(x, b, 0, range(c.lens[b])) for x in (c.k, c.v))
        o, x, o_tol, x_tol = attend(q[b, :1].cpu(), k, v, c.dim ** -0.5, torch.ones(1, c.lens[b], dtype=torch.bool))
        assert abs(lse[b, 0].cpu().double() - x[0]) <= x_tol[0] and ((out[b, 0].cpu().double() - o[0]).abs() <= o_tol[0]).all()


def queries(c, heads, kind, seed=1):
    return torch.randn(len(c.lens), heads, c.dim, generator=torch.Generator().manual_seed(seed)).to(kind)


@pytest.mark.parametrize("page", [1, 7, 16, 32, 100])
@pytest.mark.parametrize("kind,heads,kv_heads,dim", [(BF16, 4, 2, 128), (F16, 7, 1, 64), (BF16, 3, 3, 80), (F16, 2, 1, 256)])
def test_decode(ibp, kind, heads, kv_heads, dim, page):
    c = Cache(kind, kv_heads, dim, [0, 1, 31, 32, 33, 127, 128, 129, 515], page, seed=page)
    q = queries(c, heads, kind)
    before = torch.rand(len(c.lens), kv_heads, 520)
    out, lse, after = decode(ibp, c, q, before)
    check_decode(c, q, out, lse, before, after)
    plain, plain_lse, _ = decode(ibp, c, q)
    assert torch.equal(plain, out) and torch.equal(plain_lse, lse)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (16, 1), (17, 1), (40, 2), (8, 8)])
def test_decode_head_groups(ibp, heads, kv_heads):
    c = Cache(BF16, kv_heads, 64, [70, 300], 16, seed=heads)
    q = queries(c, heads, BF16)
    before = torch.zeros(2, kv_heads, 300)
    out, lse, after = decode(ibp, c, q, before)
    check_decode(c, q, out, lse, before, after)


@pytest.mark.parametrize("dim", [8, 24, 40, 72, 96, 104, 136, 192, 248])
def test_decode_head_dims(ibp, dim):
    c = Cache(F16, 2, dim, [70, 200], 16, seed=dim)
    q = queries(c, 4, F16)
    out, lse, _ = decode(ibp, c, q)
    check_decode(c, q, out, lse)


def test_decode_long(ibp):
    """A cache that is split over many blocks, alone and beside short ones."""
    for lens in ([9001], [9001, 3, 4000]):
        c = Cache(BF16, 1, 128, lens, 64, seed=2)
        q = queries(c, 4, BF16)
        before = torch.rand(len(lens), 1, 9001)
        out, lse, after = decode(ibp, c, q, before)
        check_decode(c, q, out, lse, before, after)


def test_decode_max_len_beyond_the_lengths(ibp):
    """max_len is a bound: what is split differently agrees within the bounds, lengths outside are clamped."""
    c = Cache(BF16, 2, 64, [100, 260], 16, seed=3)
    q = queries(c, 4, BF16)
    wide = torch.cat([c.table, torch.zeros(2, 200, dtype=torch.int32)], 1)
    out, lse, _ = decode(ibp, c, q, table=wide, max_len=3000)
    check_decode(c, q, out, lse)
    out, lse, _ = decode(ibp, c, q, max_len=260, lens=[100, 1 << 30])
    check_decode(c, q, out, lse)
    out, lse, _ = decode(ibp, c, q, max_len=260, lens=[100, -7])
    c.lens[1] = 0
    check_decode(c, q, out, lse)


def test_decode_absent_pages(ibp):
    """Slots of pages outside the pool count as absent, in the middle and at the end."""
    c = Cache(BF16, 2, 64, [200, 64, 30], 16, seed=4)
    q = queries(c, 4, BF16)
    table = c.table.clone()
    table[0, 3], table[0, 12], table[1, 0] = -1, 1 << 30, c.k.shape[0]
    table[2, :2] = -5
    before = torch.rand(3, 2, 200)
    out, lse, after = decode(ibp, c, q, before, table=table)
    slots = [[i for i in range(200) if i // 16 not in (3, 12)], list(range(16, 64)), []]
    check_decode(c, q, out, lse, before, after, slots)


def test_decode_nonfinite_values_reach_only_their_own(ibp):
    """A value of infinity or NaN in the cache shows in its own column, and in no other sequence."""
    c = Cache(BF16, 1, 128, [150, 150], 16, seed=5)
    q = queries(c, 4, BF16)
    clean, clean_lse, _ = decode(ibp, c, q)
    for bad in (float("inf"), float("-inf"), NAN):
        v = c.v.clone()
        v[c.table[0, 5].item(), 0, 3, 9] = bad
        out, lse, _ = decode(ibp, c, q, v=v.cuda())
        assert torch.equal(lse, clean_lse) and torch.equal(out[1], clean[1])
        other = torch.arange(128) != 9
        assert torch.equal(out[0][:, other], clean[0][:, other])
        assert torch.isnan(out[0, :, 9]).all() if bad != bad else (out[0, :, 9].float() == bad).all()


def test_decode_layouts(ibp):
    """Pools in [page][token][head] order, keys and values interleaved, as views."""
    c = Cache(BF16, 4, 64, [90, 40], 16, seed=6)
    q = queries(c, 8, BF16)
    want, want_lse, _ = decode(ibp, c, q)
    both = torch.stack([c.k, c.v], 1).transpose(2, 3).contiguous().cuda()     # [page][k, v][token][head][dim]
    k, v = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    out, lse, _ = decode(ibp, c, q, k=k, v=v)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_decode_offsets_past_32_bits(ibp):
    """Pages so far apart that their byte offsets need more than 32 bits."""
    c = Cache(BF16, 1, 64, [100], 32, seed=7, spare=0)
    q = queries(c, 2, BF16)
    want, want_lse, _ = decode(ibp, c, q)
    n, stride = c.k.shape[0], 3 << 28                # pages 1.5 GiB apart
    pool = torch.empty((n - 1) * stride + 2 * 32 * 64, dtype=BF16, device="cuda")
    k, v = (torch.as_strided(pool, (n, 1, 32, 64), (stride, 2048, 64, 1), 2048 * i) for i in range(2))
    k.copy_(c.k.cuda())
    v.copy_(c.v.cuda())
    assert (n - 1) * stride * 2 > 1 << 32
    out, lse, _ = decode(ibp, c, q, k=k, v=v)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_decode_as_many_slots_as_there_can_be(ibp):
    """2^31 - 256 slots, the most that a call takes, all of them one row (strides of 0): every slot weighs the
    same, so lse = x + ln n and out is the value, to the bit; a split left out would show as ln of what is left
    of n, 2e-3 less."""
    n, page = (1 << 31) - 256, 1 << 24
    q, row = (torch.randn(1, 1, 8, generator=torch.Generator().manual_seed(x)).to(BF16).cuda() for x in (1, 2))
    value = torch.tensor([1.0, -2.0, 0.5, 4.0, -0.25, 8.0, 1.0, -1.0], dtype=BF16, device="cuda").view(1, 1, 8)
    k, v = (x.unsqueeze(2).expand(1, 1, page, 8) for x in (row, value))
    table, lens = torch.zeros(1, 128, dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(1, 1, device="cuda")
    ibp.ibp_attn_decode(q, k, v, table, lens, n, out, lse)
    x = (q.double() @ row.double().transpose(1, 2)).item() * 8 ** -0.5
    want = x + torch.log(torch.tensor(float(n), dtype=torch.float64)).item()
    assert torch.equal(out, value)
    assert abs(lse.item() - want) <= 2.0 ** -20 * (abs(want) + abs(x))      # a logarithm and two sums in 32 bits


@pytest.mark.parametrize("heads", [64, 1024])
def test_decode_of_many_heads_under_a_wide_bound(ibp, heads):
    """max_len is only a bound: with as large a one as there is, and so many KV heads that each block could take more
    slots than 32 bits count, a short cache is read as it is."""
    n, page, most = 100, 128, (1 << 31) - 256
    g = torch.Generator().manual_seed(heads)
    q, k, v = (torch.randn(x, heads, 64, generator=g).to(BF16) for x in (1, page, page))
    pool = [x.cuda()[None].transpose(1, 2) for x in (k, v)]              # one page
    k, v = k[:n], v[:n]
    table, lens = torch.zeros(1, 1 << 24, dtype=torch.int32, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    out, lse = torch.zeros(1, heads, 64, dtype=BF16, device="cuda"), torch.zeros(1, heads, device="cuda")
    ibp.ibp_attn_decode(q.cuda(), *pool, table, lens, most, out, lse)
    out, lse = out.cpu(), lse.cpu()
    for h in range(heads):
        o, x, o_tol, x_tol = attend(q[:, h], k[:, h], v[:, h], 64 ** -0.5, torch.ones(1, n, dtype=torch.bool))
        assert abs(lse[0, h].double() - x[0]) <= x_tol[0] and ((out[0, h].double() - o[0]).abs() <= o_tol[0]).all()


@pytest.mark.parametrize("kind", [F16, BF16])
@pytest.mark.parametrize("heads,dim,n,page", [(1, 64, 131071, 64), (64, 128, 9000, 32), (512, 64, 20000, 64), (512, 128, 6000, 32),
                                              (512, 256, 6000, 32)])
def test_decode_one_slot_above_many(ibp, kind, heads, dim, n, page):
    """One slot takes nearly all of the weight and has a value of 0; what the others, at 2^-25 to 2^-30 of its weight,
    add up to is the output. None of them may be lost, in the block of the one least of all (with many heads a
    block has the whole cache): `attend`'s bound, with float16's spacing taken at the 2^12 by which its weights are
    lifted before they are rounded."""
    g = torch.Generator().manual_seed(n)
    pages = -(-n // page)
    k, v = torch.zeros(pages, 1, page, dim, dtype=kind), torch.zeros(pages, 1, page, dim, dtype=kind)
    rows_k, rows_v = k.view(-1, dim), v.view(-1, dim)
    rows_k[:, 1:] = torch.randn(rows_k.shape[0], dim - 1, generator=g).to(kind)       # (not seen by q)
    rows_k[:, 0] = -(17.5 + 3.5 * torch.rand(rows_k.shape[0], generator=g)).to(kind)
    rows_v[:] = (0.5 + torch.rand(rows_v.shape, generator=g)).to(kind)
    at = n // 3
    rows_k[at, 0], rows_v[at] = 0.0, 0.0
    q = torch.zeros(1, 1, dim, dtype=kind)
    q[0, 0, 0] = 1.0
    out, lse = torch.zeros(1, heads, dim, dtype=kind, device="cuda"), torch.zeros(1, heads, device="cuda")
    table, lens = torch.arange(pages, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda")
    ibp.ibp_attn_decode(q.cuda().expand(1, heads, dim), *(x.cuda().expand(-1, heads, -1, -1) for x in (k, v)), table, lens, n,
                        out, lse, scale=1.0)
    assert torch.equal(out, out[:, :1].expand_as(out)) and torch.equal(lse, lse[:, :1].expand_as(lse))
    o, x, o_tol, x_tol = attend(q[:, 0], rows_k[:n], rows_v[:n], 1.0, torch.ones(1, n, dtype=torch.bool))
    if kind == F16:
        o_tol -= 2.0 ** -24 * (1 - 2.0 ** -12) * rows_v[:n].double().sum(0)
    assert abs(lse.cpu()[0, 0].double() - x[0]) <= x_tol[0]
    off = (out.cpu()[0, 0].double() - o[0]).abs()
    assert (off <= o_tol[0]).all(), (off / o[0]).max()


@pytest.mark.parametrize("falling", [False, True])
@pytest.mark.parametrize("kind", [F16, BF16])
def test_decode_scores_of_millions(ibp, kind, falling):
    """Scores from 0 to 6.5 million in steps of thousands: the largest takes all, whatever the reference was before."""
    n = 1024
    k, v = (torch.randn(n // 16, 1, 16, 64, generator=torch.Generator().manual_seed(x)).to(kind) for x in (1, 2))
    scores = torch.arange(n, dtype=torch.float32) * 64
    k.view(n, 64)[:, 0] = (scores.flip(0) if falling else scores).to(kind)
    q = torch.zeros(1, 1, 64, dtype=kind, device="cuda")
    q[..., 0] = 1.0
    out, lse = torch.zeros_like(q), torch.zeros(1, 1, device="cuda")
    table, lens = torch.arange(n // 16, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda")
    ibp.ibp_attn_decode(q, k.cuda(), v.cuda(), table, lens, n, out, lse, scale=100.0)
    top = k.view(n, 64)[:, 0].max()
    best = (k.view(n, 64)[:, 0] == top).nonzero()[:, 0]                  # (bfloat16 has several of the largest)
    want, tol = v.view(n, 64)[best].double().mean(0), 2.0 ** (-10 if kind == F16 else -7)
    assert ((out[0, 0].cpu().double() - want).abs() <= tol * v.view(n, 64)[best].double().abs().mean(0) + 2.0 ** -24).all()
    assert abs(lse.item() - top.item() * 100.0) <= 2.0 ** -21 * top.item() * 100.0 + len(best)


@pytest.mark.parametrize("scale", [1e7, 1e9, 1e20, 1e30])
@pytest.mark.parametrize("kind,dim", [(BF16, 64), (F16, 64), (F16, 256)])
def test_decode_largest_scales(ibp, kind, dim, scale):
    """Scores of any size that 32 bits hold: where one slot is so far above the next that the rest weighs nothing, and no
    rounding of a score matters, its value is the output (to the rounding of its weight and of the output), and it
    has a weight of 1 more than before."""
    c = Cache(kind, 2, dim, [1, 40, 3000, 129], 16, seed=11)
    q = queries(c, 4, kind)
    before = torch.zeros(4, 2, 3000)
    out, lse, after = decode(ibp, c, q, before, scale=scale)
    checked = 0
    for b, n in enumerate(c.lens):
        for h in range(4):
            k, v = (c.rows(x, b, h // 2, range(n)) for x in (c.k, c.v))
            s = k.double() @ q[b, h].double()
            two = s.topk(min(2, n)).values
            rounding = (k.double().abs() @ q[b, h].double().abs()).max() * dim * 2.0 ** -22
            if n > 1 and ((two[0] - two[1]) * scale <= 200 or two[0] - two[1] <= rounding):
                continue
            want = v[s.argmax()].double()
            assert ((out[b, h].double() - want).abs() <= 2.02 * UNIT[kind] * want.abs() + 2.0 ** -24).all()
            assert abs(lse[b, h].item() - two[0].item() * scale) <= 2.0 ** -16 * abs(two[0].item() * scale)
            before[b, h // 2, s.argmax()] += 1
            checked += 1
    assert checked == 16 and (after - before).abs().max() <= 2.0 ** -20


@pytest.mark.parametrize("heads", [1, 512])
@pytest.mark.parametrize("sign", [1, -1])
def test_decode_of_the_largest_values(ibp, heads, sign):
    """float16 values of 65504: so is their mean, whatever the rounding of the weights (all but one 2^-11 up) makes of
    it. Infinities stay what they are."""
    n = 4096
    k, v = (torch.zeros(n // 64, 1, 64, 64, dtype=F16) for _ in range(2))
    k.view(n, 64)[:, 0] = -1.0                       # with the scale a weight of 0.50025
    k.view(n, 64)[::32, 0] = 0.0
    v[:] = sign * 65504.0
    v.view(n, 64)[n // 2 + 1, 5] = sign * float("inf")
    q = torch.zeros(1, 1, 64, dtype=F16, device="cuda")
    q[..., 0] = 1.0
    out, lse = torch.zeros(1, heads, 64, dtype=F16, device="cuda"), torch.zeros(1, heads, device="cuda")
    table, lens = torch.arange(n // 64, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda")
    ibp.ibp_attn_decode(q.expand(1, heads, 64), *(x.cuda().expand(-1, heads, -1, -1) for x in (k, v)), table, lens, n, out, lse, scale=0.69265)
    rest = torch.arange(64) != 5
    assert (out[..., rest].float() == sign * 65504.0).all() and (out[..., 5].float() == sign * float("inf")).all()


def test_decode_with_one_workspace_for_all_sizes(ibp):
    """The workspace of the most sequences and the largest max_len serves every smaller call, on both sides of the
    sizes at which the number of splits falls, with the result that a workspace of its own gives."""
    c = Cache(BF16, 8, 64, [300, 1, 170], 16, seed=9)
    q = queries(c, 8, BF16).cuda()
    k, v = c.k.cuda(), c.v.cuda()
    table = torch.cat([c.table, torch.zeros(3, 600, dtype=torch.int32)], 1).cuda()
    lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(3, 8, device="cuda")
    for weights in (False, True):
        space = torch.empty(ibp.ibp_attn_decode_workspace(3, 8, 8, 64, 9000, weights), dtype=torch.uint8, device="cuda")
        for n in (1, 2, 3):
            for m in (300, 384, 385, 4095, 5461, 5462, 8191, 8192, 8193, 8999, 9000):
                results = []
                for w in (space, None):
                    total = torch.zeros(n, 8, m, device="cuda") if weights else None
                    ibp.ibp_attn_decode(q[:n], k, v, table[:n], lens[:n], m, out[:n], lse[:n], weights=total, workspace=w)
                    results.append((out[:n].clone(), lse[:n].clone(), total))
                assert all(a is None or torch.equal(a, b) for a, b in zip(*results))
                check_decode_head(c, q, *results[0][:2])


# ---------------------------------------------------------------- eviction

def run_evict(ibp, c, weights, positions, next_positions, budget, recent, in_place=False, max_len=None):
    k, v = c.k.cuda(), c.v.cuda()
    w, p = weights.cuda(), positions.cuda()
    new_w, new_p = (w, p) if in_place else (torch.full_like(w, 7.0), torch.full_like(p, 7))
    lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    new_lens = lens if in_place else torch.full_like(lens, -1)
    nxt = torch.tensor(next_positions, dtype=torch.int32, device="cuda")
    for _ in range(1 if in_place else 2):            # (again from the same arrays gives the same)
        ibp.ibp_kv_evict(k, v, c.table.cuda(), lens, max(c.lens) if max_len is None else max_len, budget, recent, nxt, w, p,
                         new_w, new_p, new_lens)
    return k.cpu(), v.cpu(), new_w.cpu(), new_p.cpu(), new_lens.cpu()


def same(a, b):
    """Equal to the bit (NaN too)."""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def check_evict(c, weights, positions, next_positions, budget, recent, got, in_place=False):
    k, v, new_w, new_p, new_lens = got
    want = evict(weights, positions, c.lens, next_positions, budget, recent)
    for b, n in enumerate(c.lens):
        m = min(n, budget)
        assert new_lens[b] == m
        for h in range(c.kv_heads):
            of = torch.tensor(want[b][h], dtype=torch.long)
            assert same(new_w[b, h, :m], weights[b, h, of]) and torch.equal(new_p[b, h, :m], positions[b, h, of])
            if not in_place:
                assert (new_w[b, h, m:] == 7).all() and (new_p[b, h, m:] == 7).all()
            for new, old in ((k, c.k), (v, c.v)):
                assert same(c.rows(new, b, h, range(m)), c.rows(old, b, h, of))
                assert same(c.rows(new, b, h, range(m, n)), c.rows(old, b, h, range(m, n)))
    used = torch.zeros(c.k.shape[0], dtype=torch.bool)
    used[c.table.flatten().long()] = True
    assert same(k[~used], c.k[~used]) and same(v[~used], c.v[~used])


def arrays(c, seed=0, scattered=True):
    g = torch.Generator().manual_seed(seed)
    n = max(c.lens)
    weights = torch.randn(len(c.lens), c.kv_heads, n, generator=g).mul_(2).exp_()
    positions = torch.zeros(len(c.lens), c.kv_heads, n, dtype=torch.int32)
    for b, length in enumerate(c.lens):
        for h in range(c.kv_heads):
            p = torch.randperm(length, generator=g) if scattered else torch.arange(length)
            positions[b, h, :length] = p.to(torch.int32)
    return weights, positions


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (40, 0), (40, 10), (40, 40), (99, 5), (100, 0), (1000, 1000)])
def test_evict(ibp, budget, recent, in_place):
    c = Cache(BF16, 2, 64, [100, 0, 41, 40, 39, 1], 16, seed=budget)
    weights, positions = arrays(c, seed=recent)
    got = run_evict(ibp, c, weights, positions, c.lens, budget, recent, in_place)
    check_evict(c, weights, positions, c.lens, budget, recent, got, in_place)


@pytest.mark.parametrize("kind,dim,page,n,budget", [(F16, 8, 7, 2500, 1100), (BF16, 80, 24, 1025, 1024), (F16, 256, 32, 1300, 9),
                                                    (BF16, 128, 16, 5000, 2048)])
def test_evict_sizes(ibp, kind, dim, page, n, budget):
    c = Cache(kind, 1, dim, [n], page, seed=n)
    weights, positions = arrays(c, scattered=n % 2 == 0)
    got = run_evict(ibp, c, weights, positions, [n], budget, budget // 4)
    check_evict(c, weights, positions, [n], budget, budget // 4, got)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,budget", [(4096, 4000), (4097, 7), (32768, 20000), (32769, 32700), (40000, 1)])
def test_evict_long(ibp, n, budget, in_place):
    """Lengths on both sides of what is held in registers, weights of few values beside many ties."""
    c = Cache(BF16, 2, 8, [70, 3], 256, seed=1)      # (its rows are set below: two long heads are slow to draw one by one)
    c.lens, c.per = [n, n - 1000], -(-n // 256)
    c.k, c.v = (torch.randn(2 * c.per, 2, 256, 8, generator=torch.Generator().manual_seed(i)).to(BF16) for i in (1, 2))
    c.table = torch.randperm(2 * c.per, generator=torch.Generator().manual_seed(3)).view(2, c.per).to(torch.int32)
    weights, positions = arrays(c, seed=budget)
    weights[0, 1] = (weights[0, 1] * 2).round()
    got = run_evict(ibp, c, weights, positions, c.lens, budget, budget // 3, in_place)
    check_evict(c, weights, positions, c.lens, budget, budget // 3, got, in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n", [4095, 4096, 4097, 16383, 16384, 16385, 36863, 36864, 36865])
def test_evict_at_the_limits_of_what_lds_holds(ibp, n, in_place):
    """Keys are held in LDS, in arrays of 4,096, 16,384 and 36,864, and above that computed again: the last slot of
    each and the first beyond it, kept and dropped; one slot too many, and nearly all of them."""
    c = Cache(BF16, 1, 8, [1, 1], 256, seed=1)       # (its rows are set below)
    c.lens, c.per = [n, n - 3], -(-n // 256)
    c.k, c.v = (torch.randn(2 * c.per, 1, 256, 8, generator=torch.Generator().manual_seed(i)).to(BF16) for i in (1, 2))
    c.table = torch.randperm(2 * c.per, generator=torch.Generator().manual_seed(3)).view(2, c.per).to(torch.int32)
    for budget, recent, last in ((n - 1, 7, 0.0), (n - 1, 0, 1e9), (100, 3, 1e9)):
        weights, positions = arrays(c, seed=n)
        weights[0, 0, -1] = weights[1, 0, n - 4] = last
        positions[0, 0, -1] = positions[1, 0, n - 4] = -1              # (not kept for its position)
        got = run_evict(ibp, c, weights, positions, c.lens, budget, recent, in_place)
        check_evict(c, weights, positions, c.lens, budget, recent, got, in_place)


def test_evict_ties_and_special_weights(ibp):
    """Equal weights go by the lowest slot; NaN ranks as -inf, -0 as 0, infinities where they belong."""
    c = Cache(BF16, 3, 64, [300, 300], 16, seed=1)
    weights, positions = arrays(c)
    weights[0] = 1.0
    weights[1, 0] = (weights[1, 0] > 1).float()
    weights[1, 1, ::3], weights[1, 1, 1::7], weights[1, 1, 2::11] = NAN, NEG, float("inf")
    weights[1, 2] = torch.tensor([0.0, -0.0]).repeat(150)
    weights[1, 2, 250:] = -torch.rand(50)
    for budget in (10, 100, 299):
        got = run_evict(ibp, c, weights, positions, c.lens, budget, 7)
        check_evict(c, weights, positions, c.lens, budget, 7, got)


def test_evict_layout_and_positions_beyond(ibp):
    """[page][token][head] pools; positions of a long conversation whose older tokens are gone."""
    c = Cache(BF16, 2, 64, [80, 64], 16, seed=3)
    weights, positions = arrays(c)
    positions = positions * 1000 + 5
    nxt = [79 * 1000 + 6, 2 ** 31 - 1]
    both = torch.stack([c.k, c.v], 1).transpose(2, 3).contiguous().cuda()
    k, v = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    lens = torch.tensor(c.lens, dtype=torch.int32, device="cuda")
    new_w, new_p, new_lens = torch.full((2, 2, 32), 7.0, device="cuda"), torch.full((2, 2, 32), 7, dtype=torch.int32, device="cuda"), torch.zeros_like(lens)
    ibp.ibp_kv_evict(k, v, c.table.cuda(), lens, 80, 32, 32, torch.tensor(nxt, dtype=torch.int32, device="cuda"), weights.cuda(),
                     positions.cuda(), new_w, new_p, new_lens)
    check_evict(c, weights, positions, nxt, 32, 32, (k.cpu(), v.cpu(), new_w.cpu(), new_p.cpu(), new_lens.cpu()))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,budget", [(40, 39), (400, 200)])
def test_evict_from_an_empty_pool(ibp, n, budget, in_place):
    """A pool without pages holds no tokens: nothing is moved, new lengths are 0 and the rest stays."""
    k, v = (torch.empty(0, 2, 16, 64, dtype=BF16, device="cuda") for _ in range(2))
    table = torch.zeros(1, -(-n // 16), dtype=torch.int32, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    weights, positions = torch.rand(1, 2, n, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda").repeat(1, 2, 1)
    new_w, new_p = torch.full((1, 2, budget), 7.0, device="cuda"), torch.full((1, 2, budget), 7, dtype=torch.int32, device="cuda")
    new_lens = lens if in_place else torch.full_like(lens, 7)
    ibp.ibp_kv_evict(k, v, table, lens, n, budget, 3, lens.clone(), weights, positions, new_w, new_p, new_lens)
    assert new_lens.tolist() == [0] and bool((new_w == 7).all()) and bool((new_p == 7).all())


def test_decode_then_evict_in_a_graph(ibp):
    """A serving step captured into a graph and replayed with the program's own work between: every replay
    equals the same calls made one by one."""
    c = Cache(BF16, 2, 128, [300, 280], 32, seed=8)
    q = queries(c, 8, BF16).cuda()
    weights, positions = arrays(c, seed=5)

    def state():
        return dict(k=c.k.cuda(), v=c.v.cuda(), w=weights.cuda(), new_w=torch.zeros(2, 2, 256, device="cuda"),
                    new_p=torch.zeros(2, 2, 256, dtype=torch.int32, device="cuda"),
                    new_lens=torch.zeros(2, dtype=torch.int32, device="cuda"),
                    out=torch.zeros_like(q), lse=torch.zeros(2, 8, device="cuda"))

    table, lens, pos = c.table.cuda(), torch.tensor(c.lens, dtype=torch.int32, device="cuda"), positions.cuda()
    space = torch.empty(ibp.ibp_attn_decode_workspace(2, 8, 2, 128, 300, True), dtype=torch.uint8, device="cuda")
    space2 = torch.empty(ibp.ibp_kv_evict_workspace(2, 2, 300, 256), dtype=torch.uint8, device="cuda")

    def step(s):
        ibp.ibp_attn_decode(q, s["k"], s["v"], table, lens, 300, s["out"], s["lse"], weights=s["w"], workspace=space)
        ibp.ibp_kv_evict(s["k"], s["v"], table, lens, 300, 256, 64, lens, s["w"], pos, s["new_w"], s["new_p"], s["new_lens"],
                         workspace=space2)

    eager, s = state(), state()
    graph = torch.cuda.CUDAGraph()
    step(state())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(s)
    for _ in range(4):
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        q.mul_(1)                                    # (work of the program's own on the stream)
        torch.cuda.synchronize()
        for name in eager:
            assert same(eager[name], s[name]), name


def test_paged_calls_refuse(ibp):
    c = Cache(BF16, 2, 64, [40], 16)
    q, k, v, table = queries(c, 4, BF16).cuda(), c.k.cuda(), c.v.cuda(), c.table.cuda()
    lens, out = torch.tensor([40], dtype=torch.int32, device="cuda"), torch.empty(1, 4, 64, dtype=BF16, device="cuda")
    args = dict(q=q, k=k, v=v, table=table, lens=lens, max_len=40, out=out)
    for error, status, bad in [
            (TypeError, None, dict(k=k.half())), (TypeError, None, dict(q=q.half())), (ValueError, None, dict(v=v[:1])),
            (TypeError, None, dict(table=table.long())), (ValueError, None, dict(table=table[0])), (ValueError, None, dict(lens=lens[:0])),
            (TypeError, None, dict(lens=lens.cpu())), (ValueError, None, dict(out=out[:, :2])), (ValueError, None, dict(weights=out)),
            (ibp.IbpError, ibp.IBP_ERANGE, dict(max_len=49)), (ibp.IbpError, ibp.IBP_EINVAL, dict(scale=-1.0)),
            (ibp.IbpError, ibp.IBP_EINVAL, dict(q=q[:, :3], out=out[:, :3])),
            (ibp.IbpError, ibp.IBP_ENOMEM, dict(weights=torch.zeros(1, 2, 39, device="cuda"))),
            (ibp.IbpError, ibp.IBP_ENOMEM, dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"),
                                                weights=torch.zeros(1, 2, 40, device="cuda")))]:
        with pytest.raises(error) as e:
            ibp.ibp_attn_decode(**{**args, **bad})
        assert status is None or e.value.status == status
    w, p = (x.cuda() for x in arrays(c))
    args = dict(k=k, v=v, table=table, lens=lens, max_len=40, budget=20, recent=5, next_positions=lens, weights=w, positions=p,
                new_weights=w, new_positions=p, new_lens=lens)
    small = torch.zeros(1, 2, 19, device="cuda")
    for error, status, bad in [
            (ibp.IbpError, ibp.IBP_EINVAL, dict(budget=0)), (ibp.IbpError, ibp.IBP_EINVAL, dict(recent=21)),
            (ibp.IbpError, ibp.IBP_ERANGE, dict(max_len=49)), (ValueError, None, dict(positions=p[:, :1])),
            (TypeError, None, dict(positions=p.long())), (TypeError, None, dict(weights=w.double())),
            (ibp.IbpError, ibp.IBP_ENOMEM, dict(new_weights=small, new_positions=small.int())),
            (ibp.IbpError, ibp.IBP_EINVAL, dict(weights=w[..., :39].contiguous(), positions=p[..., :39].contiguous())),
            (ibp.IbpError, ibp.IBP_ENOMEM, dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")))]:
        with pytest.raises(error) as e:
            ibp.ibp_kv_evict(**{**args, **bad})
        assert status is None or e.value.status == status
