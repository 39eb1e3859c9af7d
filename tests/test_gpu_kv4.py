"""A cache of 4-bit records: reading its rows, attention of single tokens over it, eviction from it, and all of them together."""
import pytest
import torch

from attention_reference import NEG, U32, attend, evict
from kv_reference import attend4, parts_of, record_bytes, records_of, rotation_table, turn, values_of, weights4

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ibp():
    import paper_2605_30728_amd
    return paper_2605_30728_amd


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """A paged cache of records on the CPU, its pages in no order; all bits set (codes of 15, NaN) outside the lengths."""

    def __init__(self, kind, kv_heads, dim, lens, page, seed=0, spare=3, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.lens, self.page, self.kv_heads, self.dim = kind, list(lens), page, kv_heads, dim
        self.per = max(-(-max(lens) // page), 1)
        n, width = len(lens) * self.per + spare, record_bytes(dim)
        self.keys, self.values = (torch.full((n, kv_heads, page, width), 255, dtype=torch.uint8) for _ in range(2))
        self.table = torch.randperm(n, generator=g)[:len(lens) * self.per].view(len(lens), self.per).to(torch.int32)
        for b, length in enumerate(lens):
            if length == 0:
                continue
            slot = torch.arange(length)
            at = self.table[b, slot // page].long(), slice(None), slot % page
            for pool in (self.keys, self.values):
                x = torch.randn(length, kv_heads, dim, generator=g) * spread
                x[..., ::17] *= 6
                pool[at] = records_of(x.to(kind).float(), kind)

    def rows(self, pool, b, h, slots):
        slots = torch.as_tensor(slots, dtype=torch.long)
        return pool[self.table[b].long()[slots // self.page], h, slots % self.page]


def queries(c, heads, seed=1):
    return torch.randn(len(c.lens), heads, c.dim, generator=torch.Generator().manual_seed(seed)).to(c.kind)


def decode(ibp, c, q, weights=None, max_len=None, keys=None, values=None, scale=None, lens=None, table=None, **more):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    w = None if weights is None else weights.cuda()
    ibp.ibp_attn_decode4(q.cuda(), c.keys.cuda() if keys is None else keys, c.values.cuda() if values is None else values,
                         (c.table if table is None else table).cuda(), int32(c.lens if lens is None else lens),
                         max(c.lens) if max_len is None else max_len, out, lse, weights=w, scale=scale, **more)
    return out.cpu(), lse.cpu(), None if w is None else w.cpu()


def check(c, q, out, lse, before=None, after=None, slots=None, scale=None):
    group = q.shape[1] // c.kv_heads
    scale = c.dim ** -0.5 if scale is None else scale
    for b in range(q.shape[0]):
        at = list(range(c.lens[b])) if slots is None else slots[b]
        for g in range(c.kv_heads):
            k, v = c.rows(c.keys, b, g, at), c.rows(c.values, b, g, at)
            added, tol = torch.zeros(len(at), dtype=torch.float64), torch.zeros(len(at), dtype=torch.float64)
            for h in range(g * group, (g + 1) * group):
                o, x, o_tol, x_tol = attend4(q[b, h], k, v, scale)
                assert (lse[b, h] == NEG) == (x == NEG)
                assert x == NEG or abs(lse[b, h].double() - x) <= x_tol
                off = (out[b, h].double() - o).abs()
                assert (off <= o_tol).all(), (b, h, (off / o_tol.clamp(min=1e-30)).max())
                if at and before is not None:
                    w, w_tol = weights4(q[b, h], k, scale)
                    added, tol = added + w, tol + w_tol
            if before is not None:
                want = before[b, g, at].double() + added
                assert ((after[b, g, at].double() - want).abs() <= tol + added * group * 2.0 ** -24 + want * 2.0 ** -23).all()
                rest = torch.ones(before.shape[2], dtype=torch.bool)
                rest[at] = False
                assert torch.equal(after[b, g, rest], before[b, g, rest])


# ---------------------------------------------------------------- reading

@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("dim", [8, 24, 40, 64, 96, 128, 200, 256])
@pytest.mark.parametrize("page", [1, 7, 32])
def test_read(ibp, kind, dim, page):
    """Bit for bit what the records stand for, and the rows behind a history as they were."""
    c = Cache(kind, 3, dim, [0, 1, 33, 70], page, seed=dim)
    rows = [2, 1, 40, 70]
    starts = [sum(rows[:i]) for i in range(5)]
    k, v = (torch.full((starts[-1] + 2, 3, dim), 7.0, dtype=kind, device="cuda") for _ in range(2))
    ibp.ibp_kv4_read(c.keys.cuda(), c.values.cuda(), c.table.cuda(), int32(c.lens), k, v, int32(starts))
    for pool, got in ((c.keys, k.cpu()), (c.values, v.cpu())):
        want = torch.full_like(got, 7.0)
        for b, n in enumerate(c.lens):
            for h in range(3):
                want[starts[b]:starts[b] + n, h] = values_of(c.rows(pool, b, h, range(n)), dim, kind, torch.float32).to(kind)
        assert torch.equal(got, want)


@pytest.mark.parametrize("kind,kv_heads,dim", [(BF16, 8, 128), (F16, 17, 40), (BF16, 3, 256)])
def test_read_many_rows(ibp, kind, kv_heads, dim):
    c = Cache(kind, kv_heads, dim, [1500, 0, 700], 24, seed=dim)
    k, v = (torch.full((2201, kv_heads, dim), 7.0, dtype=kind, device="cuda") for _ in range(2))
    ibp.ibp_kv4_read(c.keys.cuda(), c.values.cuda(), c.table.cuda(), int32(c.lens), k, v, int32([0, 1500, 1500, 2200]))
    for pool, got in ((c.keys, k.cpu()), (c.values, v.cpu())):
        want = torch.full_like(got, 7.0)
        for b, first, n in ((0, 0, 1500), (2, 1500, 700)):
            for h in range(kv_heads):
                want[first:first + n, h] = values_of(c.rows(pool, b, h, range(n)), dim, kind, torch.float32).to(kind)
        assert torch.equal(got, want)


def test_read_from_a_slot_on(ibp):
    """`first`, fewer rows than slots, absent pages, a row per sequence, and numbers outside everything."""
    c = Cache(BF16, 2, 64, [50, 64, 30], 16, seed=2)
    table = c.table.clone()
    table[1, 1] = -1
    pools = c.keys.cuda(), c.values.cuda()
    first, rows, starts = [45, 10, -3], [9, 40, 6], [0, 9, 49, 55]
    k, v = (torch.full((55, 2, 64), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    ibp.ibp_kv4_read(*pools, table.cuda(), int32(c.lens), k, v, int32(starts), int32(first))
    for pool, got in ((c.keys, k.cpu()), (c.values, v.cpu())):
        want = torch.full_like(got, 7.0)
        for b in range(3):
            for i in range(rows[b]):
                slot = first[b] + i
                if 0 <= slot < c.lens[b] and not (b == 1 and slot // 16 == 1):
                    for h in range(2):
                        want[starts[b] + i, h] = values_of(c.rows(pool, b, h, [slot]), 64, BF16, torch.float32).to(BF16)[0]
        assert torch.equal(got, want)
    k1, v1 = (torch.full((3, 2, 64), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    ibp.ibp_kv4_read(*pools, c.table.cuda(), int32(c.lens), k1, v1, first=int32([49, 1 << 30, 0]))
    assert torch.equal(k1[0].cpu(), torch.stack([values_of(c.rows(c.keys, 0, h, [49]), 64, BF16, torch.float32).to(BF16)[0] for h in range(2)]))
    assert (k1[1] == 7.0).all() and (v1[1] == 7.0).all() and not (v1[2] == 7.0).all()
    k[:], starts = 7.0, [-4, 1 << 30, 5, 9]                               # (starts that make no sense: nothing out of bounds)
    ibp.ibp_kv4_read(*pools, c.table.cuda(), int32(c.lens), k, v, int32(starts))
    torch.cuda.synchronize()


# ---------------------------------------------------------------- attention

@pytest.mark.parametrize("page", [1, 7, 16, 64, 100])
@pytest.mark.parametrize("kind,heads,kv_heads,dim", [(BF16, 4, 2, 128), (F16, 7, 1, 64), (BF16, 3, 3, 80), (F16, 2, 1, 256), (F16, 4, 2, 128)])
def test_decode(ibp, kind, heads, kv_heads, dim, page):
    c = Cache(kind, kv_heads, dim, [0, 1, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 515], page, seed=page)
    q = queries(c, heads)
    before = torch.rand(len(c.lens), kv_heads, 520)
    out, lse, after = decode(ibp, c, q, before)
    check(c, q, out, lse, before, after)
    plain, plain_lse, _ = decode(ibp, c, q)
    assert torch.equal(plain, out) and torch.equal(plain_lse, lse)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (16, 1), (17, 1), (40, 2), (8, 8)])
def test_decode_head_groups(ibp, heads, kv_heads):
    c = Cache(BF16, kv_heads, 64, [70, 300], 16, seed=heads)
    q = queries(c, heads)
    before = torch.zeros(2, kv_heads, 300)
    out, lse, after = decode(ibp, c, q, before)
    check(c, q, out, lse, before, after)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("dim", [8, 24, 32, 40, 72, 96, 104, 136, 160, 192, 224, 248])
def test_decode_head_dims(ibp, dim, kind):
    c = Cache(kind, 2, dim, [70, 200], 16, seed=dim)
    q = queries(c, 4)
    out, lse, _ = decode(ibp, c, q)
    check(c, q, out, lse)


@pytest.mark.parametrize("lens", [[9001], [9001, 3, 4000], [20000]])
def test_decode_long(ibp, lens):
    c = Cache(BF16, 1, 128, lens, 64, seed=2)
    q = queries(c, 4)
    before = torch.rand(len(lens), 1, max(lens))
    out, lse, after = decode(ibp, c, q, before)
    check(c, q, out, lse, before, after)


def test_decode_max_len_beyond_the_lengths(ibp):
    c = Cache(BF16, 2, 64, [100, 260], 16, seed=3)
    q = queries(c, 4)
    wide = torch.cat([c.table, torch.zeros(2, 200, dtype=torch.int32)], 1)
    out, lse, _ = decode(ibp, c, q, table=wide, max_len=3000)
    check(c, q, out, lse)
    out, lse, _ = decode(ibp, c, q, max_len=260, lens=[100, 1 << 30])
    check(c, q, out, lse)
    out, lse, _ = decode(ibp, c, q, max_len=260, lens=[100, -7])
    c.lens[1] = 0
    check(c, q, out, lse)


def test_decode_absent_pages(ibp):
    c = Cache(BF16, 2, 64, [200, 64, 30], 16, seed=4)
    q = queries(c, 4)
    table = c.table.clone()
    table[0, 3], table[0, 12], table[1, 0] = -1, 1 << 30, c.keys.shape[0]
    table[2, :2] = -5
    before = torch.rand(3, 2, 200)
    out, lse, after = decode(ibp, c, q, before, table=table)
    slots = [[i for i in range(200) if i // 16 not in (3, 12)], list(range(16, 64)), []]
    check(c, q, out, lse, before, after, slots)
    none = c.keys[:0].cuda()
    out, lse, after = decode(ibp, c, q, before, keys=none, values=none)
    assert (out == 0).all() and (lse == NEG).all() and torch.equal(after, before)


@pytest.mark.parametrize("kind", [BF16, F16])
def test_decode_groups_of_nan(ibp, kind):
    """Of a value: its own 32 columns, in its own sequence; of a key: its own head."""
    c = Cache(kind, 2, 128, [150, 150], 16, seed=5)
    q = queries(c, 4)
    clean, clean_lse, _ = decode(ibp, c, q)
    nan = torch.tensor([float("nan")], dtype=kind).view(torch.uint8)
    for at in (64, 72):                              # the step, then the centre of group 1
        v = c.values.clone()
        v[c.table[0, 5].long(), 0, 3, at + 2:at + 4] = nan
        out, lse, _ = decode(ibp, c, q, values=v.cuda())
        rest = (torch.arange(128) < 32) | (torch.arange(128) >= 64)
        assert torch.equal(lse, clean_lse) and torch.equal(out[1], clean[1]) and torch.equal(out[0, 2:], clean[0, 2:])
        assert torch.equal(out[0, :2][:, rest], clean[0, :2][:, rest]) and out[0, :2][:, ~rest].isnan().all()
        k = c.keys.clone()
        k[c.table[0, 5].long(), 0, 3, at + 2:at + 4] = nan
        out, lse, _ = decode(ibp, c, q, keys=k.cuda())
        assert lse[0, :2].isnan().all() and out[0, :2].isnan().all()
        assert torch.equal(lse[1], clean_lse[1]) and torch.equal(out[0, 2:], clean[0, 2:]) and torch.equal(out[1], clean[1])


@pytest.mark.parametrize("kind", [BF16, F16])
def test_decode_queries_that_are_not_finite(ibp, kind):
    """Their own heads' results are NaN, and no other's."""
    c = Cache(kind, 2, 128, [150, 90], 16, seed=18)
    q = queries(c, 8)
    before = torch.rand(2, 2, 150)
    clean, clean_lse, clean_w = decode(ibp, c, q, before)
    for bad in (float("inf"), float("-inf"), float("nan")):
        x = q.clone()
        x[0, 1, 77] = bad
        out, lse, w = decode(ibp, c, x, before)
        assert out[0, 1].isnan().all() and lse[0, 1].isnan()
        rest = torch.ones(2, 8, dtype=torch.bool)
        rest[0, 1] = False
        assert torch.equal(out[rest], clean[rest]) and torch.equal(lse[rest], clean_lse[rest])
        assert torch.equal(w[1], clean_w[1]) and torch.equal(w[0, 1], clean_w[0, 1])


def test_two_streams_at_once(ibp):
    """Two decodes with workspaces of their own, and an append, on streams of their own: each as alone."""
    c = [Cache(BF16, 2, 128, [3000, 500], 32, seed=s) for s in (19, 20)]
    q = [queries(x, 8, s).cuda() for s, x in enumerate(c)]
    tensors = [(x.keys.cuda(), x.values.cuda(), x.table.cuda(), int32(x.lens)) for x in c]
    want = [decode(ibp, x, y.cpu()) for x, y in zip(c, q)]
    streams = [torch.cuda.Stream() for _ in c]
    outs = [(torch.zeros_like(y), torch.zeros(2, 8, device="cuda")) for y in q]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, y, s, (o, lse) in zip(tensors, q, streams, outs):
            ibp.ibp_attn_decode4(y, *x, 3000, o, lse, stream=s)
    torch.cuda.synchronize()
    for (o, lse), w in zip(outs, want):
        assert torch.equal(o.cpu(), w[0]) and torch.equal(lse.cpu(), w[1])


def test_decode_layouts(ibp):
    c = Cache(BF16, 4, 64, [90, 40], 16, seed=6)
    q = queries(c, 8)
    want, want_lse, _ = decode(ibp, c, q)
    both = torch.stack([c.keys, c.values], 1).transpose(2, 3).contiguous().cuda()
    out, lse, _ = decode(ibp, c, q, keys=both[:, 0].transpose(1, 2), values=both[:, 1].transpose(1, 2))
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    wide = torch.zeros(2, 8, 72, dtype=BF16)
    wide[..., :64] = q
    out = torch.full((2, 8, 80), 7.0, dtype=BF16, device="cuda")
    ibp.ibp_attn_decode4(wide.cuda()[..., :64], c.keys.cuda(), c.values.cuda(), c.table.cuda(), int32(c.lens), 90, out[..., :64])
    assert torch.equal(out[..., :64].cpu(), want) and (out[..., 64:] == 7.0).all()


def test_decode_offsets_past_32_bits(ibp):
    c = Cache(BF16, 1, 64, [100], 32, seed=7, spare=0)
    q = queries(c, 2)
    want, want_lse, _ = decode(ibp, c, q)
    n, stride = c.keys.shape[0], 3 << 29
    pool = torch.empty((n - 1) * stride + 2 * 32 * 48, dtype=torch.uint8, device="cuda")
    k, v = (torch.as_strided(pool, (n, 1, 32, 48), (stride, 1536, 48, 1), 1536 * i) for i in range(2))
    k.copy_(c.keys.cuda())
    v.copy_(c.values.cuda())
    out, lse, _ = decode(ibp, c, q, keys=k, values=v)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_decode_as_many_slots_as_there_can_be(ibp):
    """2^31 - 256 slots, the most that a call takes, all of them one record (strides of 0): lse = x + ln n and the output is what the
    record stands for; a split left out would show as ln of what is left of n, 2e-3 less."""
    n, page = (1 << 31) - 256, 1 << 24
    g = torch.Generator().manual_seed(1)
    q = torch.randn(1, 1, 32, generator=g).to(BF16)
    record = records_of(torch.randn(2, 32, generator=g).to(BF16).float(), BF16)
    pools = [x.view(1, 1, 1, 32).cuda().expand(1, 1, page, 32) for x in record]
    table = torch.zeros(1, 128, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros(1, 1, 32, dtype=BF16, device="cuda"), torch.zeros(1, 1, device="cuda")
    ibp.ibp_attn_decode4(q.cuda(), *pools, table, int32([n]), n, out, lse)
    x = (q[0, 0].double() @ values_of(record[0], 32, BF16)).item() * 32 ** -0.5
    want = x + torch.log(torch.tensor(float(n), dtype=torch.float64)).item()
    assert abs(lse.item() - want) <= 2.0 ** -19 * (abs(want) + abs(x))
    code, step, centre = parts_of(record[1], 32, BF16)
    value = code * step + centre
    # (the output's rounding, and 2^16 sums that each wave adds up for its 2^20 slots, each off by up to u32 of 55 step + |centre|)
    assert ((out[0, 0].cpu().double() - value).abs() <= 2.0 ** -8 * 1.01 * value.abs() + 2.0 ** 16 * U32 * (55 * step + centre.abs())).all()


def test_decode_of_many_heads_under_a_wide_bound(ibp):
    """max_len is only a bound: with as large a one as there is, a short cache is read as it is."""
    c = Cache(BF16, 64, 64, [100], 128, seed=17)
    q = queries(c, 64)
    out, lse, _ = decode(ibp, c, q, table=torch.cat([c.table, torch.zeros(1, (1 << 24) - 1, dtype=torch.int32)], 1), max_len=(1 << 31) - 256)
    check(c, q, out, lse)


@pytest.mark.parametrize("kind", [F16, BF16])
@pytest.mark.parametrize("heads,n", [(1, 131071), (64, 9000), (512, 6000)])
def test_decode_one_slot_above_many(ibp, kind, heads, n):
    """One slot takes nearly all of the weight and has a value of 0; what the others, at 2^-25 to 2^-30 of its weight, add up
    to is the output, to the bound of their own rounding."""
    g = torch.Generator().manual_seed(n)
    pages, dim = -(-n // 64), 64
    k, v = torch.zeros(pages * 64, dim), 0.5 + torch.rand(pages * 64, dim, generator=g)
    k[:, :32] = -(17.5 + 3.5 * torch.rand(pages * 64, 1, generator=g)) / 32
    at = n // 3
    k[at], v[at] = 0.0, 0.0
    keys, values = (records_of(x.to(kind).float(), kind) for x in (k, v))
    q = torch.zeros(1, 1, dim, dtype=kind)
    q[..., :32] = 1.0
    pools = [x.view(pages, 1, 64, 48).cuda().expand(-1, heads, -1, -1) for x in (keys, values)]
    out, lse = torch.zeros(1, heads, dim, dtype=kind, device="cuda"), torch.zeros(1, heads, device="cuda")
    ibp.ibp_attn_decode4(q.cuda().expand(1, heads, dim), *pools, torch.arange(pages, dtype=torch.int32, device="cuda")[None], int32([n]), n, out,
                         lse, scale=1.0)
    assert torch.equal(out, out[:, :1].expand_as(out)) and torch.equal(lse, lse[:, :1].expand_as(lse))
    o, x, o_tol, x_tol = attend4(q[0, 0], keys[:n], values[:n], 1.0)
    assert abs(lse[0, 0].cpu().double() - x) <= x_tol
    assert ((out[0, 0].cpu().double() - o).abs() <= o_tol).all()


@pytest.mark.parametrize("scale", [1e4, 1e9, 1e20, 1e30])
@pytest.mark.parametrize("kind,dim", [(BF16, 64), (F16, 128)])
def test_decode_largest_scales(ibp, kind, dim, scale):
    """Where one slot is so far above the next that no rounding matters, its value is the output, to its rounding and the
    weight's (that of its step, and the output's)."""
    c = Cache(kind, 2, dim, [1, 40, 3000, 129], 16, seed=11)
    q = queries(c, 4)
    before = torch.zeros(4, 2, 3000)
    out, lse, after = decode(ibp, c, q, before, scale=scale)
    checked = 0
    for b, n in enumerate(c.lens):
        for h in range(4):
            keys, values = (c.rows(x, b, h // 2, range(n)) for x in (c.keys, c.values))
            _, step, centre = parts_of(keys, dim, kind)
            s = values_of(keys, dim, kind) @ q[b, h].double()
            rounding = ((55 * step + centre.abs()) @ q[b, h].double().abs()).max() * (dim + 24) * U32
            two, best = s.topk(min(2, n)).values, s.argmax().item()
            if n > 1 and ((two[0] - two[1]) * scale <= 200 or two[0] - two[1] <= 2 * rounding):
                continue
            want, _, tol, _ = attend4(q[b, h], keys[best:best + 1], values[best:best + 1], 1e-30)
            assert ((out[b, h].double() - want).abs() <= tol).all()
            assert abs(lse[b, h].item() - two[0].item() * scale) <= (rounding.item() + 2.0 ** -20 * abs(two[0].item())) * scale
            before[b, h // 2, best] += 1
            checked += 1
    assert checked >= 14


def test_decode_extreme_records(ibp):
    """Steps and centres at the ends of the types, queries of very small and large values."""
    for kind, small, large in ((BF16, 1e-30, 1e30), (F16, 2e-5, 2e4)):
        for spread in (small, large):
            c = Cache(kind, 1, 64, [100, 7], 16, seed=8, spread=spread / 20)
            q = queries(c, 2)
            out, lse, _ = decode(ibp, c, q, scale=1 / max(spread, 1e-4))
            check(c, q, out, lse, scale=1 / max(spread, 1e-4))
        c = Cache(kind, 1, 64, [100, 7], 16, seed=9)
        q = (queries(c, 2).float() * (1e-3 if kind == F16 else 1e-20)).to(kind)
        out, lse, _ = decode(ibp, c, q, scale=1e3 if kind == F16 else 1e19)
        check(c, q, out, lse, scale=1e3 if kind == F16 else 1e19)
        q[..., 0] = 1000.0
        out, lse, _ = decode(ibp, c, q, scale=1e-3)
        check(c, q, out, lse, scale=1e-3)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("falling", [False, True])
def test_decode_steps_of_all_sizes(ibp, kind, falling):
    """Values a thousand times larger at one end of a cache than at the other, groups a hundred times larger than others, slots
    without a step: what the steps are taken relative to changes on the way."""
    c = Cache(kind, 2, 128, [2000, 300], 32, seed=15)
    g = torch.Generator().manual_seed(2)
    for b, n in enumerate(c.lens):
        slot = torch.arange(n)
        size = 10.0 ** (4 * slot / n - 2)
        x = torch.randn(n, 2, 128, generator=g) * (size.flip(0) if falling else size)[:, None, None]
        x[..., 32:64] *= 100 if kind == BF16 else 0.01
        x[::7, :, 64:96] = x[::7, :, 64:65]
        c.values[c.table[b, slot // 32].long(), :, slot % 32] = records_of(x.to(kind).float(), kind)
    q = queries(c, 4)
    before = torch.rand(2, 2, 2000)
    out, lse, after = decode(ibp, c, q, before)
    check(c, q, out, lse, before, after)


def test_decode_infinite_step(ibp):
    """Of one group in a bfloat16 cache: its columns are not finite, all others as without it."""
    c = Cache(BF16, 1, 64, [300], 16, seed=16)
    q = queries(c, 2)
    clean, _, _ = decode(ibp, c, q)
    v = c.values.clone()
    v[c.table[0, 9].long(), 0, 5, 32:34] = torch.tensor([float("inf")], dtype=BF16).view(torch.uint8)
    out, _, _ = decode(ibp, c, q, values=v.cuda())
    assert not out[0, :, :32].isfinite().any() and torch.equal(out[0, :, 32:], clean[0, :, 32:])


def test_decode_one_workspace_serves_smaller_calls(ibp):
    c = Cache(BF16, 2, 128, [300, 5000, 40], 32, seed=10)
    q = queries(c, 8)
    space = torch.empty(ibp.ibp_attn_decode4_workspace(3, 8, 2, 128, 5000, True), dtype=torch.uint8, device="cuda")
    for n, most in ((3, 5000), (2, 4097), (1, 300), (1, 129)):
        d = Cache(BF16, 2, 128, [min(x, most) for x in c.lens[:n]], 32, seed=10)
        space.fill_(255)
        before = torch.rand(n, 2, most)
        out, lse, after = decode(ibp, d, q[:n], before, max_len=most, table=torch.cat([d.table, torch.zeros(n, 200, dtype=torch.int32)], 1), workspace=space)
        check(d, q[:n], out, lse, before, after)


def test_decode_repeats(ibp):
    c = Cache(F16, 2, 128, [5000, 1, 777], 32, seed=12)
    q = queries(c, 8)
    before = torch.rand(3, 2, 5000)
    first = decode(ibp, c, q, before)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, decode(ibp, c, q, before)))


# ---------------------------------------------------------------- together

def test_evict_moves_records(ibp):
    """ibp_kv_evict over the pools seen as rows of record / 2 16-bit values: what is kept keeps its records."""
    c = Cache(BF16, 2, 128, [80, 33], 16, seed=13)
    g = torch.Generator().manual_seed(1)
    weights = torch.rand(2, 2, 80, generator=g)
    positions = torch.arange(80, dtype=torch.int32).repeat(2, 2, 1)
    k, v, w, p, lens = c.keys.cuda(), c.values.cuda(), weights.cuda(), positions.cuda(), int32(c.lens)
    ibp.ibp_kv_evict(k.view(BF16), v.view(BF16), c.table.cuda(), lens, 80, 40, 8, int32(c.lens), w, p, w, p, lens)
    for b, heads in enumerate(evict(weights, positions, c.lens, c.lens, 40, 8)):
        for h, source in enumerate(heads):
            m = len(source)
            assert lens[b] == m and torch.equal(p[b, h, :m].cpu(), positions[b, h, source])
            for pool, now in ((c.keys, k.cpu()), (c.values, v.cpu())):
                assert torch.equal(c.rows(now, b, h, range(m)), c.rows(pool, b, h, source))


@pytest.mark.parametrize("kind", [BF16, F16])
def test_a_run_of_all_of_them(ibp, kind):
    """Two turns of prompts and tokens in between over a 4-bit cache held at a budget: append, read for the prompt's attention, decode
    with weights, evict; each result against the definition of what the cache held."""
    heads, kv_heads, dim, page, budget, recent = 6, 2, 64, 16, 60, 10
    per, n = 10, 3
    g = torch.Generator().manual_seed(3)
    width = record_bytes(dim)
    c = Cache(kind, kv_heads, dim, [0, 0, 0], page)
    c.per = per
    c.table = torch.randperm(n * per, generator=g).view(n, per).to(torch.int32)
    keys, values = (torch.full((n * per, kv_heads, page, width), 255, dtype=torch.uint8, device="cuda") for _ in range(2))
    weights = torch.zeros(n, kv_heads, per * page, device="cuda")
    positions = torch.zeros(n, kv_heads, per * page, dtype=torch.int32, device="cuda")
    lens, nxt, table, rotation = int32([0] * n), int32([0] * n), c.table.cuda(), rotation_table(400, dim // 2).cuda()
    random = lambda rows, h: torch.randn(rows, h, dim, generator=g).to(kind).cuda()  # noqa: E731

    def turn_of(new):
        old = lens.tolist()
        lens.add_(int32(new))
        nxt.add_(int32(new))
        starts = int32([sum(new[:i]) for i in range(n + 1)])
        k_starts = int32([sum(a + b for a, b in list(zip(old, new))[:i]) for i in range(n + 1)])
        q, k, v = random(sum(new), heads), random(sum(new), kv_heads), random(sum(new), kv_heads)
        ibp.ibp_kv4_append(k, v, keys, values, table, lens, nxt, starts, rotation, q=q, weights=weights, positions=positions)
        all_k, all_v = (torch.full((sum(old) + sum(new), kv_heads, dim), 7.0, dtype=kind, device="cuda") for _ in range(2))
        ibp.ibp_kv4_read(keys, values, table, lens, all_k, all_v, k_starts)
        out = torch.empty_like(q)
        lse = torch.empty(heads, q.shape[0], device="cuda")
        ibp.ibp_attn_prompt(q, all_k, all_v, starts, k_starts, out, lse)
        got = torch.zeros(kv_heads, all_k.shape[0], device="cuda")
        ibp.ibp_attn_key_weights(q, all_k, starts, k_starts, lse, got)
        for b in range(n):
            m = int(lens[b])
            weights[b, :, :m] += got[:, int(k_starts[b]):int(k_starts[b]) + m]
        # every sequence's last row sees all of its cache
        c.keys, c.values, c.lens = keys.cpu(), values.cpu(), lens.tolist()
        for b in range(n):
            if new[b] == 0:
                continue
            row = int(starts[b + 1]) - 1
            for h in range(heads):
                at = slice(int(k_starts[b]), int(k_starts[b + 1]))
                o, x, tol, x_tol = attend(q[row:row + 1, h].cpu(), all_k[at, h // 3].cpu(), all_v[at, h // 3].cpu(), dim ** -0.5,
                                          torch.ones(1, c.lens[b], dtype=torch.bool))
                assert ((out[row, h].cpu().double() - o[0]).abs() <= tol[0]).all()
                held = [values_of(c.rows(pool, b, h // 3, range(c.lens[b])), dim, kind, torch.float32).to(kind) for pool in (c.keys, c.values)]
                assert torch.equal(all_k[at, h // 3].cpu(), held[0]) and torch.equal(all_v[at, h // 3].cpu(), held[1])

    def token():
        lens.add_(1)
        nxt.add_(1)
        q, k, v = random(n, heads), random(n, kv_heads), random(n, kv_heads)
        ibp.ibp_kv4_append(k, v, keys, values, table, lens, nxt, rotation=rotation, q=q, weights=weights, positions=positions)
        before = weights.cpu()
        out, lse = torch.empty_like(q), torch.empty(n, heads, device="cuda")
        ibp.ibp_attn_decode4(q, keys, values, table, lens, per * page, out, lse, weights=weights)
        c.keys, c.values, c.lens = keys.cpu(), values.cpu(), lens.tolist()
        check(c, q.cpu(), out.cpu(), lse.cpu(), before, weights.cpu())
        for b in range(n):                           # the newest key is the turned one
            angles = rotation[int(nxt[b]) - 1].cpu()
            want = records_of(turn(k[b].cpu(), angles, True, torch.float32), kind)
            got = torch.stack([c.rows(c.keys, b, h, [c.lens[b] - 1])[0] for h in range(kv_heads)])
            assert torch.equal(got[:, :40], want[:, :40])
            assert (positions[b, :, c.lens[b] - 1] == int(nxt[b]) - 1).all()

    def hold():
        ibp.ibp_kv_evict(keys.view(BF16), values.view(BF16), table, lens, per * page, budget, recent, nxt, weights, positions, weights,
                         positions, lens)
        for b in range(n):
            m = int(lens[b])
            assert m <= budget
            for h in range(kv_heads):
                assert len(set(positions[b, h, :m].tolist())) == m

    turn_of([50, 1, 0])
    for _ in range(3):
        token()
    turn_of([20, 0, 70])
    hold()
    for _ in range(4):
        token()
        hold()
    assert nxt.tolist() == [77, 8, 77] and lens.tolist() == [60, 8, 60]


def test_a_step_in_a_graph(ibp):
    """Append and decode captured together and replayed over a growing cache: every replay as the eager calls."""
    c = Cache(BF16, 2, 128, [200, 31, 64], 16, seed=14)
    table, rotation = c.table.cuda(), rotation_table(300, 64).cuda()
    g = torch.Generator().manual_seed(4)
    keys, values = c.keys.cuda(), c.values.cuda()
    lens = int32(c.lens)
    q, k, v = (torch.zeros(3, h, 128, dtype=BF16, device="cuda") for h in (8, 2, 2))
    turned, out, weights = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(3, 2, 208, device="cuda")
    space = torch.empty(ibp.ibp_attn_decode4_workspace(3, 8, 2, 128, 208, True), dtype=torch.uint8, device="cuda")

    def step(pools, w, o):
        ibp.ibp_kv4_append(k, v, *pools, table, lens, lens, rotation=rotation, q=q, q_out=turned, weights=w)
        ibp.ibp_attn_decode4(turned, *pools, table, lens, 208, o, weights=w, workspace=space)

    twin, twin_w, twin_out = (keys.clone(), values.clone()), weights.clone(), torch.zeros_like(out)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step((keys, values), weights, out)
    for i in range(6):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g).to(BF16))
        lens.add_(1)
        graph.replay()
        step(twin, twin_w, twin_out)
        torch.cuda.synchronize()
        assert torch.equal(out, twin_out) and torch.equal(weights, twin_w) and torch.equal(keys, twin[0]) and torch.equal(values, twin[1])


def test_refusals(ibp):
    c = Cache(BF16, 2, 64, [40], 16)
    q = queries(c, 4).cuda()
    keys, values, table, lens = c.keys.cuda(), c.values.cuda(), c.table.cuda(), int32(c.lens)
    base = dict(q=q, keys=keys, values=values, table=table, lens=lens, max_len=40, out=torch.empty_like(q))
    for error, bad in [(TypeError, dict(q=q.float())), (TypeError, dict(keys=keys.view(BF16))), (ValueError, dict(keys=keys[..., :32])),
                       (ValueError, dict(values=values[:1])), (TypeError, dict(table=table.long())), (ValueError, dict(lens=lens[:0])),
                       (TypeError, dict(out=q.half())), (ValueError, dict(out=q[:, :2])), (ValueError, dict(q=q[:0])),
                       (ibp.IbpError, dict(max_len=1000)), (ValueError, dict(max_len=-1)), (ibp.IbpError, dict(q=q[:, :3], out=q[:, :3])),
                       (ValueError, dict(weights=torch.zeros(1, 3, 40, device="cuda"))), (TypeError, dict(lse=torch.zeros(1, 4, device="cuda", dtype=F16))),
                       (ibp.IbpError, dict(weights=torch.zeros(1, 2, 39, device="cuda"))),
                       (ibp.IbpError, dict(weights=torch.zeros(1, 2, 40, device="cuda"), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))),
                       (ibp.IbpError, dict(scale=0.0)), (ibp.IbpError, dict(scale=1e39)), (ibp.IbpError, dict(scale=float("nan")))]:
        with pytest.raises(error):
            ibp.ibp_attn_decode4(**{**base, **bad})
    rows = torch.empty(40, 2, 64, dtype=BF16, device="cuda")
    base = dict(keys=keys, values=values, table=table, lens=lens, k=rows, v=rows.clone(), starts=int32([0, 40]))
    for error, bad in [(TypeError, dict(k=rows.float())), (ValueError, dict(v=rows[:, :1])), (ValueError, dict(keys=keys[..., :32])),
                       (ValueError, dict(starts=None)), (ValueError, dict(starts=int32([0]))), (TypeError, dict(first=lens.long())),
                       (ValueError, dict(first=lens[:0])), (TypeError, dict(table=c.table))]:
        with pytest.raises(error):
            ibp.ibp_kv4_read(**{**base, **bad})
    ibp.ibp_kv4_read(**base)
