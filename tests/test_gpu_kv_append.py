"""New rows into a paged cache of 16-bit values and of 4-bit records, against their definitions."""
import pytest
import torch

from attention_reference import UNIT
from kv_reference import (held_bound, record_bytes, records_of, rotation_table, turn, turn_bound, values_of)

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ibp():
    import paper_2605_30728_amd
    return paper_2605_30728_amd


class Case:
    """Sequences that hold `held` slots and get `new` rows each; pools filled with a pattern."""

    def __init__(self, kind, heads, kv_heads, dim, turned, halves, new, held, page=16, gone=0, after=0, seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.kind, self.heads, self.kv_heads, self.dim, self.turned, self.halves, self.page = kind, heads, kv_heads, dim, turned, halves, page
        self.new, self.held, self.n = list(new), list(held), len(new)
        rows = sum(new) + after
        self.q, self.k, self.v = ((torch.randn(rows, h, dim, generator=g) * spread).to(kind) for h in (heads, kv_heads, kv_heads))
        self.lens = [a + b for a, b in zip(new, held)]
        self.next = [x + gone for x in self.lens]
        per = max(max(-(-x // page) for x in self.lens), 1)
        self.n_pages = self.n * per + 2
        self.table = torch.randperm(self.n_pages, generator=g)[:self.n * per].view(self.n, per).to(torch.int32)
        self.rotation = rotation_table(max(max(self.next), 1), turned // 2)
        self.slots = max(max(self.lens), 1) + 3

    def pools(self, four):
        if four:
            return [torch.full((self.n_pages, self.kv_heads, self.page, record_bytes(self.dim)), 0xA5 + i, dtype=torch.uint8) for i in range(2)]
        return [torch.full((self.n_pages, self.kv_heads, self.page, self.dim), 7.0 + i, dtype=self.kind) for i in range(2)]

    def places(self):
        """(row, sequence, slot, position) of every row of a sequence."""
        row = 0
        for b, n in enumerate(self.new):
            for i in range(n):
                yield row, b, self.held[b] + i, self.next[b] - n + i
                row += 1


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts_of(new):
    return int32([sum(new[:i]) for i in range(len(new) + 1)])


def append(ibp, c, four=False, q=True, in_place=False, pools=None, table=None, lens=None, next_positions=None, starts=True, tracked=True,
           rotation=True, **more):
    """The call; what it left, on the CPU."""
    pools = [x.cuda() for x in (c.pools(four) if pools is None else pools)]
    qs = c.q.cuda()
    out = qs if in_place else torch.full_like(qs, 5.0)
    w = torch.full((c.n, c.kv_heads, c.slots), 3.0, device="cuda")
    p = torch.full((c.n, c.kv_heads, c.slots), -9, dtype=torch.int32, device="cuda")
    (ibp.ibp_kv4_append if four else ibp.ibp_kv_append)(
        c.k.cuda(), c.v.cuda(), *pools, (c.table if table is None else table).cuda(), int32(c.lens if lens is None else lens),
        int32(c.next if next_positions is None else next_positions), starts=starts_of(c.new) if starts else None,
        rotation=c.rotation.cuda() if rotation and c.turned else None, halves=c.halves, q=qs if q else None,
        q_out=out if q and not in_place else None, weights=w if tracked else None, positions=p if tracked else None, **more)
    return [x.cpu() for x in (*pools, out, w, p)]


def near(got, x, angles, c):
    """A turned row against its definition."""
    want = turn(x, angles, c.halves)
    tol = turn_bound(x, angles, c.halves) + UNIT[c.kind] * want.abs() * 1.01 + (2.0 ** -24 if c.kind == F16 else 0)
    rest = torch.arange(c.dim) >= 2 * angles.shape[0]
    assert torch.equal(got[:, rest], x[:, rest])
    assert ((got.double() - want).abs() <= tol).all()


def check(c, four, keys, values, out, w, p, missing=(), q=True, tracked=True, queries=None, clamp=None):
    """Every row where it belongs, and everything else as it was; `missing`: rows that are not appended."""
    want_k, want_v = c.pools(four)
    want_w, want_p = torch.full_like(w, 3.0), torch.full_like(p, -9)
    seen = torch.zeros(c.q.shape[0], dtype=torch.bool)
    for row, b, slot, position in c.places():
        angles = c.rotation[min(max(position, 0), c.rotation.shape[0] - 1)]
        if q:
            near(out[row], c.q[row], angles, c)
            seen[row] = True
        if row in missing:
            continue
        at = c.table[b, slot // c.page].item(), slice(None), slot % c.page
        if four:
            rows = torch.stack([turn(c.k[row], angles, c.halves, torch.float32), c.v[row].float()])
            want_k[at], want_v[at] = records_of(rows, c.kind)
            n = 20 * -(-c.dim // 32)                                     # (the padding stays)
            want_k[at][:, n:], want_v[at][:, n:] = 0xA5, 0xA6
            exact = torch.stack([turn(c.k[row], angles, c.halves), c.v[row].double()])
            got = torch.stack([keys[at], values[at]])
            ok = exact.isfinite().unflatten(-1, (-1, 8)).all(-1, keepdim=True).expand(*exact.shape[:-1], -1, 8).flatten(-2)
            off = (values_of(got, c.dim, c.kind) - exact).abs()
            assert ((off <= held_bound(exact, got, c.kind) + (2.0 ** -21 if c.kind == F16 else 0)) | ~ok | off.isnan()).all()
        else:
            near(keys[at], c.k[row], angles, c)
            want_k[at], want_v[at] = keys[at], c.v[row]
        if tracked:
            want_w[b, :, slot], want_p[b, :, slot] = 0.0, position
    assert torch.equal(keys.view(torch.uint8), want_k.view(torch.uint8)) and torch.equal(values.view(torch.uint8), want_v.view(torch.uint8))
    assert torch.equal(w, want_w) and torch.equal(p, want_p)
    assert (out[~seen] == (5.0 if queries is None else queries[~seen])).all()


FOUR = pytest.mark.parametrize("four", [False, True], ids=["16bit", "4bit"])


@FOUR
@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("dim,turned,halves", [(8, 8, True), (8, 8, False), (24, 8, True), (40, 40, True), (64, 64, False), (64, 32, True),
                                               (72, 72, True), (80, 80, True), (96, 48, False), (128, 128, True), (128, 0, True),
                                               (136, 136, False), (192, 64, True), (248, 248, True), (256, 256, True)])
def test_head_dims(ibp, four, kind, dim, turned, halves):
    c = Case(kind, 6, 2, dim, turned, halves, [3, 0, 1, 18], [5, 40, 0, 14], gone=11, after=2, seed=dim)
    check(c, four, *append(ibp, c, four))


@FOUR
@pytest.mark.parametrize("page", [1, 7, 16, 100])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (32, 8), (16, 16), (28, 4)])
def test_pages_and_heads(ibp, four, heads, kv_heads, page):
    c = Case(BF16, heads, kv_heads, 64, 64, True, [33, 2], [0, 95], page=page, seed=page)
    check(c, four, *append(ibp, c, four))


@FOUR
def test_one_row_per_sequence(ibp, four):
    """Without starts; the same as with them."""
    c = Case(BF16, 8, 2, 128, 128, True, [1] * 70, [7 * i % 50 for i in range(70)], gone=3)
    with_starts = append(ibp, c, four)
    check(c, four, *with_starts)
    assert all(torch.equal(a, b) for a, b in zip(with_starts, append(ibp, c, four, starts=False)))


@FOUR
@pytest.mark.parametrize("n", [1, 63, 64, 65, 130, 5000])
def test_many_sequences(ibp, four, n):
    """Empty ones among them, at the start and the end too."""
    new = [0 if i % 3 != 1 else 1 + i % 4 for i in range(n)]
    c = Case(F16, 2, 1, 32, 16, False, new, [i % 6 for i in range(n)], after=3)
    check(c, four, *append(ibp, c, four))


@FOUR
def test_no_queries_no_rotation_nothing_tracked(ibp, four):
    c = Case(BF16, 4, 2, 96, 96, True, [5, 9], [0, 3])
    c.turned, c.rotation = 0, torch.zeros(20, 0, 2)
    check(c, four, *append(ibp, c, four, q=False, tracked=False), q=False, tracked=False)


@FOUR
@pytest.mark.parametrize("halves", [True, False])
def test_queries_in_place(ibp, four, halves):
    c = Case(BF16, 32, 2, 128, 96, halves, [40, 3], [1, 0], after=1)
    check(c, four, *append(ibp, c, four, in_place=True), queries=c.q)


@FOUR
def test_rows_that_have_no_slot(ibp, four):
    """A negative slot, one beyond the table, absent pages: not appended, the query is turned all the same. Positions
    beyond the table of angles take its last, or first."""
    c = Case(BF16, 4, 2, 64, 64, True, [20, 20, 20], [0, 20, 0], seed=3)
    c.slots = 50
    lens, nxt, table = list(c.lens), list(c.next), c.table.clone()
    lens[0] = 15                                     # rows 0 .. 4 have negative slots
    lens[1] = 60                                     # rows 28 .. 39 are beyond the table's 48 slots
    table[2, 0] = -1                                 # rows 40 .. 55
    table[0, 2] = 1 << 30                            # (no row's)
    nxt[1], nxt[2] = 1000, 10                        # positions 980 .. 999 and -10 .. 9, of 40 angles
    got = append(ibp, c, four, table=table, lens=lens, next_positions=nxt)
    c.held, c.next, c.table = [-5, 40, 0], nxt, table
    check(c, four, *got, missing={*range(5), *range(28, 56)})


@FOUR
def test_slots_beyond_the_tracked_ones(ibp, four):
    """Their rows are appended, weights and positions have no place for them."""
    c = Case(BF16, 4, 2, 64, 64, True, [20], [10], seed=3)
    want = append(ibp, c, four)
    c.slots = 25
    got = append(ibp, c, four)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(got[3], want[3][..., :25]) and torch.equal(got[4], want[4][..., :25])


@FOUR
def test_an_empty_pool_takes_nothing(ibp, four):
    c = Case(BF16, 4, 2, 64, 64, True, [4], [0])
    pools = [x[:0] for x in c.pools(four)]
    keys, values, out, w, p = append(ibp, c, four, pools=pools)
    assert (w == 3.0).all() and (p == -9).all()
    for row, _, _, position in c.places():
        near(out[row], c.q[row], c.rotation[position], c)


@FOUR
def test_an_empty_pool_without_a_table(ibp, four):
    """Nothing is looked up: a null table is allowed where there are no pages."""
    from paper_2605_30728_amd import attention as at
    c = Case(BF16, 4, 2, 64, 64, True, [4], [0])
    k, v, q, out, rotation, lens, starts = c.k.cuda(), c.v.cuda(), c.q.cuda(), c.q.cuda(), c.rotation.cuda(), int32(c.lens), starts_of(c.new)
    rows = lambda x: at.ibp_rows(x.data_ptr(), x.shape[0], x.stride(0), x.stride(1))  # noqa: E731
    from paper_2605_30728_amd.kv_cache import ibp_rotation
    pages = at.ibp_pages(None, None, 0, 16, 3, None, *[0] * 6)
    status = getattr(ibp.lib(), "ibp_kv4_append" if four else "ibp_kv_append")(
        at.ibp_attn(0, 4, 2, 64, 1.0, 0), rows(k), rows(v), rows(q), rows(out), ibp_rotation(rotation.data_ptr(), rotation.shape[0], 64, 1),
        starts.data_ptr(), 1, pages, lens.data_ptr(), lens.data_ptr(), None, None, 0, torch.cuda.current_stream().cuda_stream)
    assert status == ibp.IBP_OK
    torch.cuda.synchronize()
    for row, _, _, position in c.places():
        near(out[row].cpu(), c.q[row], c.rotation[position], c)
    if four:
        assert ibp.lib().ibp_kv4_read(at.ibp_attn(0, 2, 2, 64, 1.0, 0), pages, lens.data_ptr(), 1, starts.data_ptr(), None, rows(k), rows(v),
                                      torch.cuda.current_stream().cuda_stream) == ibp.IBP_OK
        torch.cuda.synchronize()
        assert torch.equal(k.cpu(), c.k) and torch.equal(v.cpu(), c.v)


@FOUR
@pytest.mark.parametrize("kind,heads,kv_heads,dim,turned,halves", [(BF16, 32, 8, 128, 128, True), (F16, 28, 4, 80, 48, True),
                                                                   (BF16, 17, 17, 40, 40, False), (F16, 6, 3, 256, 256, True)])
def test_calls_of_many_rows(ibp, four, kind, heads, kv_heads, dim, turned, halves):
    """Several items of every lane on their way; heads that do not fill the last part of a row."""
    c = Case(kind, heads, kv_heads, dim, turned, halves, [700, 0, 3, 1500], [1, 5, 20, 0], page=24, gone=7, after=1, seed=heads)
    check(c, four, *append(ibp, c, four))


@FOUR
def test_layouts(ibp, four):
    """Rows as views of one projection, pools in [page][token][head] order, keys and values interleaved."""
    c = Case(BF16, 6, 2, 64, 64, True, [9, 30], [2, 0], seed=5)
    want = append(ibp, c, four)
    one = torch.cat([c.q, c.k, c.v], 1).cuda()
    q, k, v = one.split([6, 2, 2], 1)
    a, b = c.pools(four)
    both = torch.stack([a, b], 1).transpose(2, 3).contiguous().cuda()
    keys, values = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    wide = torch.full((c.q.shape[0], 6, 72), 5.0, dtype=BF16, device="cuda")
    (ibp.ibp_kv4_append if four else ibp.ibp_kv_append)(k, v, keys, values, c.table.cuda(), int32(c.lens), int32(c.next), starts_of(c.new),
                                                        c.rotation.cuda(), True, q, wide[..., :64])
    assert torch.equal(keys.cpu(), want[0]) and torch.equal(values.cpu(), want[1]) and torch.equal(wide[..., :64].cpu(), want[2])
    assert (wide[..., 64:] == 5.0).all() and torch.equal(one.cpu(), torch.cat([c.q, c.k, c.v], 1))


@FOUR
def test_offsets_past_32_bits(ibp, four):
    c = Case(BF16, 2, 1, 64, 64, True, [40], [0], page=32, seed=6)
    want = append(ibp, c, four)
    n, width = c.n_pages, 64 if not four else 48
    kind, stride = (torch.uint8, 3 << 29) if four else (BF16, 3 << 28)            # pages 1.5 GiB apart
    pool = torch.empty((n - 1) * stride + 2 * 32 * width, dtype=kind, device="cuda")
    keys, values = (torch.as_strided(pool, (n, 1, 32, width), (stride, 32 * width, width, 1), 32 * width * i) for i in range(2))
    for x, y in zip((keys, values), c.pools(four)):
        x.copy_(y.cuda())
    (ibp.ibp_kv4_append if four else ibp.ibp_kv_append)(c.k.cuda(), c.v.cuda(), keys, values, c.table.cuda(), int32(c.lens), int32(c.next),
                                                        starts_of(c.new), c.rotation.cuda())
    assert torch.equal(keys.cpu(), want[0]) and torch.equal(values.cpu(), want[1])


@pytest.mark.parametrize("kind", [BF16, F16])
def test_groups_that_cannot_be_held(ibp, kind):
    """An infinity or NaN makes its group of 32 NaN, of a key or a value, and no other; equal values are held exactly; the
    type's largest values, of both signs, are held."""
    c = Case(kind, 2, 2, 128, 0, True, [8], [0])
    top = torch.finfo(kind).max
    c.k[0, 0, 5], c.k[1, 1, 100], c.v[2, 0, 40] = float("inf"), float("nan"), float("-inf")
    c.k[3], c.v[3] = 2.5, -top
    c.k[4, 0, 0], c.k[4, 0, 1] = top, -top
    c.v[5] = 0.0
    c.k[6] = torch.finfo(kind).tiny
    keys, values, out, w, p = append(ibp, c, True)
    check(c, True, keys, values, out, w, p)
    page = c.table[0, 0].long()
    held = [values_of(x[page], 128, kind) for x in (keys, values)]
    bad = torch.zeros(2, 2, 8, 128, dtype=torch.bool)
    bad[0, 0, 0, :32], bad[0, 1, 1, 96:], bad[1, 0, 2, 32:64] = True, True, True
    for x in range(2):
        assert torch.equal(held[x][:, :8].isnan(), bad[x])
    assert (held[0][:, 3] == 2.5).all() and (held[1][:, 3] == -top).all() and (held[1][:, 5] == 0).all()


@FOUR
@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("spread", [1e-4, 30.0])
def test_sizes_of_values(ibp, four, kind, spread):
    c = Case(kind, 4, 2, 128, 128, True, [60], [0], spread=spread)
    check(c, four, *append(ibp, c, four))


@FOUR
def test_on_a_stream_and_in_a_graph(ibp, four):
    """On another stream than the current one, and captured, replayed with new rows and lengths: every replay as the eager call."""
    c = Case(BF16, 8, 2, 128, 128, True, [1] * 5, [0, 3, 15, 16, 40], gone=2)
    want = append(ibp, c, four)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    pools, qs = [x.cuda() for x in c.pools(four)], c.q.cuda()
    k, v, lens, nxt, table, rotation = c.k.cuda(), c.v.cuda(), int32(c.lens), int32(c.next), c.table.cuda(), c.rotation.cuda()
    out = torch.full_like(qs, 5.0)
    call = ibp.ibp_kv4_append if four else ibp.ibp_kv_append
    torch.cuda.synchronize()
    call(k, v, *pools, table, lens, nxt, rotation=rotation, q=qs, q_out=out, stream=stream)
    stream.synchronize()
    assert torch.equal(pools[0].cpu(), want[0]) and torch.equal(pools[1].cpu(), want[1]) and torch.equal(out.cpu(), want[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(k, v, *pools, table, lens, nxt, rotation=rotation, q=qs, q_out=out)
    for i in range(4):
        g = torch.Generator().manual_seed(i)
        c.q, c.k, c.v = (torch.randn(x.shape, generator=g).to(BF16) for x in (c.q, c.k, c.v))
        c.held = [(h + 1) % 30 for h in c.held]
        c.lens, c.next = [h + 1 for h in c.held], [h + 3 for h in c.held]
        for x, y in zip((*pools, qs, k, v, lens, nxt), (*c.pools(four), c.q, c.k, c.v, int32(c.lens), int32(c.next))):
            x.copy_(y)
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        want = append(ibp, c, four)
        assert torch.equal(pools[0].cpu(), want[0]) and torch.equal(pools[1].cpu(), want[1]) and torch.equal(out.cpu(), want[2])


def test_refusals(ibp):
    c = Case(BF16, 4, 2, 64, 64, True, [4], [0])
    dev = lambda *x: [y.cuda() for y in x]  # noqa: E731
    k, v, q, table, rotation = dev(c.k, c.v, c.q, c.table, c.rotation)
    lens, starts = int32(c.lens), starts_of(c.new)
    for four, call in ((False, ibp.ibp_kv_append), (True, ibp.ibp_kv4_append)):
        pools = dev(*c.pools(four))
        base = dict(k=k, v=v, keys=pools[0], values=pools[1], table=table, lens=lens, next_positions=lens, starts=starts, rotation=rotation, q=q)
        for error, bad in [(TypeError, dict(k=c.k)), (TypeError, dict(k=k.float())), (TypeError, dict(v=v.half())), (ValueError, dict(v=v[:, :1])),
                           (ValueError, dict(keys=pools[0][:, :1])), (TypeError, dict(keys=pools[0].float())), (TypeError, dict(table=table.long())),
                           (ValueError, dict(lens=lens[:0])), (TypeError, dict(next_positions=lens.long())), (ValueError, dict(starts=None)),
                           (ValueError, dict(starts=starts[:1])), (TypeError, dict(rotation=rotation.double())), (ValueError, dict(rotation=rotation[0])),
                           (ibp.IbpError, dict(rotation=rotation[:, :3].contiguous())), (ibp.IbpError, dict(rotation=torch.zeros(9, 40, 2, device="cuda"))),
                           (ValueError, dict(q=None, q_out=q)), (ValueError, dict(q=q[..., :32])), (ibp.IbpError, dict(q=q[:, :3])),
                           (ValueError, dict(weights=torch.zeros(1, 3, 9, device="cuda"))),
                           (TypeError, dict(positions=torch.zeros(1, 2, 9, device="cuda"))),
                           (ValueError, dict(weights=torch.zeros(1, 2, 9, device="cuda"), positions=torch.zeros(1, 2, 8, dtype=torch.int32, device="cuda")))]:
            with pytest.raises(error):
                call(**{**base, **bad})
        call(**base)
