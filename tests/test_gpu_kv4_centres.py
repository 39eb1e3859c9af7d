"""Decode over 4-bit caches whose values lie in the centres of their groups.

The bound of kv_reference.attend4 counts a rounding of weights times steps alone. The weights of centres are fp32 in a float16
cache and two bfloat16 parts in a bfloat16 one: of a weight from 1 to 2 the first part leaves up to 2^-8, which a
number of 8 bits holds to 2^-17, so that 2^-17 sum p |centre| is added there.
"""
import math

import pytest
import torch

from attention_reference import NEG
from kv_reference import attend4, parts_of, records_of, weights4
from test_gpu_kv4 import Cache, decode, int32

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ibp():
    import paper_2605_30728_amd
    return paper_2605_30728_amd


def sharp(c, heads, seed, spread=1.0):
    """Keys whose first group's centre alone says how far a slot is seen, queries of one value: scores of up to a few units with
    next to no rounding of their own."""
    g = torch.Generator().manual_seed(seed)
    for b, n in enumerate(c.lens):
        slot = torch.arange(n)
        k = torch.zeros(n, c.kv_heads, c.dim)
        k[..., :32] = torch.randn(n, c.kv_heads, 1, generator=g) * spread
        c.keys[c.table[b, slot // c.page].long(), :, slot % c.page] = records_of(k.to(c.kind).float(), c.kind)
    q = torch.zeros(len(c.lens), heads, c.dim)
    q[..., 0] = 1 + torch.rand(len(c.lens), heads, generator=g)
    return q.to(c.kind)


def fill(c, values_of_slots):
    for b, n in enumerate(c.lens):
        slot = torch.arange(n)
        c.values[c.table[b, slot // c.page].long(), :, slot % c.page] = records_of(values_of_slots(n).to(c.kind).float(), c.kind)


def near(q, keys, values, out, lse, scale=1.0):
    """One query head against its definition."""
    o, x, tol, x_tol = attend4(q, keys, values, scale)
    if q.dtype == BF16:
        p, _ = weights4(q, keys, scale)
        tol = tol + 1.01 * 2.0 ** -17 * (p @ parts_of(values, q.shape[0], q.dtype)[2].abs())
    assert x != NEG and abs(lse.double() - x) <= x_tol
    off = (out.double() - o).abs()
    assert (off <= tol).all(), (off / tol.clamp(min=1e-300)).max()


def check(c, q, out, lse):
    group = q.shape[1] // c.kv_heads
    for b, n in enumerate(c.lens):
        for h in range(q.shape[1]):
            near(q[b, h], *(c.rows(x, b, h // group, range(n)) for x in (c.keys, c.values)), out[b, h], lse[b, h])


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("dim", [8, 32, 40, 64, 96, 128, 160, 200, 224, 256])
def test_groups_of_equal_values(ibp, kind, dim):
    """With signs that differ from slot to slot, so that what they add up to is far below what is added up."""
    c = Cache(kind, 2, dim, [16, 200, 3, 1000], 16, seed=dim)
    g = torch.Generator().manual_seed(dim + 1)
    groups = -(-dim // 32)
    fill(c, lambda n: torch.randn(n, 2, groups, generator=g).repeat_interleave(32, -1)[..., :dim])
    q = sharp(c, 6, dim + 2)
    out, lse, _ = decode(ibp, c, q, scale=1.0)
    check(c, q, out, lse)
    weighed, weighed_lse, _ = decode(ibp, c, q, torch.rand(4, 2, 1000), scale=1.0)
    assert torch.equal(weighed, out) and torch.equal(weighed_lse, lse)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("nearly", [2.0 ** -6, 0.1])
def test_large_means_of_both_signs(ibp, kind, nearly):
    c = Cache(kind, 2, 128, [16, 500, 64], 32, seed=4)
    g = torch.Generator().manual_seed(5)
    sign = lambda n: torch.randint(0, 2, (n, 2, 4, 1), generator=g) * 2.0 - 1  # noqa: E731
    fill(c, lambda n: (sign(n) * 10 * (1 + nearly * torch.randn(n, 2, 4, 32, generator=g))).flatten(2))
    q = sharp(c, 4, 6)
    out, lse, _ = decode(ibp, c, q, scale=1.0)
    check(c, q, out, lse)


@pytest.mark.parametrize("kind", [BF16, F16])
def test_sizes_of_centres(ibp, kind):
    """From the type's smallest numbers, those that have few bits among them, to large ones."""
    for size in (2.0 ** -133, 2.0 ** -127, 1e-30, 1e-3, 1e30) if kind == BF16 else (2.0 ** -24, 2.0 ** -16, 2.0 ** -8, 2.0 ** 14):
        c = Cache(kind, 1, 64, [40, 130], 16, seed=7)
        g = torch.Generator().manual_seed(8)
        fill(c, lambda n: (torch.randint(1, 4, (n, 1, 2, 1), generator=g) * size).expand(-1, -1, -1, 32).flatten(2))
        q = sharp(c, 2, 9)
        out, lse, _ = decode(ibp, c, q, scale=1.0)
        for b in range(2):
            o, _, tol, _ = attend4(q[b, 0], c.rows(c.keys, b, 0, range(c.lens[b])), c.rows(c.values, b, 0, range(c.lens[b])), 1.0)
            # (a bfloat16 output below 2^-126 is off by up to half of 2^-133)
            assert ((out[b, 0].double() - o).abs() <= tol + (2.0 ** -134 if kind == BF16 else 0)).all(), size
            assert (out[b, 0] > 0).all()


@pytest.mark.parametrize("steps", [False, True])
def test_values_far_above_one(ibp, steps):
    """Of a bfloat16 cache whose values add up to nearly 2^128: what they stand for is finite, and so is the result."""
    c = Cache(BF16, 2, 96, [1, 40, 130], 16, seed=10)
    g = torch.Generator().manual_seed(11)
    size = 2.0 ** 118
    if steps:
        fill(c, lambda n: torch.randn(n, 2, 96, generator=g).clamp(-3, 3) * size)
    else:
        fill(c, lambda n: (torch.randint(1, 4, (n, 2, 3, 1), generator=g) * size).expand(-1, -1, -1, 32).flatten(2))
    q = sharp(c, 4, 12)
    out, lse, _ = decode(ibp, c, q, scale=1.0)
    assert out.isfinite().all()
    check(c, q, out, lse)


def test_steps_far_below_one(ibp):
    """The smallest steps that a bfloat16 cache holds, with weights down to 2^-20: as precise as others."""
    c = Cache(BF16, 2, 64, [1, 40, 1000], 16, seed=13)
    g = torch.Generator().manual_seed(14)
    for size in (2.0 ** -124, 2.0 ** -118, 2.0 ** -112):
        fill(c, lambda n: torch.randn(n, 2, 64, generator=g) * size)
        q = sharp(c, 4, 15, 4.0)
        out, lse, _ = decode(ibp, c, q, scale=1.0)
        for b, n in enumerate(c.lens):
            for h in range(4):
                keys, values = (c.rows(x, b, h // 2, range(n)) for x in (c.keys, c.values))
                o, _, tol, _ = attend4(q[b, h], keys, values, 1.0)
                p, _ = weights4(q[b, h], keys, 1.0)
                tol = tol + 1.01 * 2.0 ** -17 * (p @ parts_of(values, 64, BF16)[2].abs())
                # (a bfloat16 output below 2^-126 is off by up to half of 2^-133, and fp32 sums of such numbers by up to half of 2^-149 each)
                assert ((out[b, h].double() - o).abs() <= tol + 2.0 ** -134 + 2 * n * 2.0 ** -150).all(), size


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("down", [25.0, 33.3, 36.3, 38.5])
@pytest.mark.parametrize("heads", [1, 512])
def test_one_slot_above_many(ibp, kind, down, heads):
    """One slot of value 0 has all of the weight but what 60,000 others, of a large centre, have at 2^-down of it each: their sum
    is the output, which the type holds. With many heads a wave has a quarter of the slots."""
    n, dim, page = 60001, 64, 64
    pages = -(-n // page)
    k, v = torch.zeros(pages * page, dim), torch.full((pages * page, dim), 60000.0)
    k[:, :32] = -down * math.log(2) / 32
    k[n // 3], v[n // 3] = 0.0, 0.0
    keys, values = (records_of(x.to(kind).float(), kind) for x in (k, v))
    q = torch.zeros(1, 1, dim, dtype=kind)
    q[..., :32] = 1.0
    out, lse = torch.zeros(1, heads, dim, dtype=kind, device="cuda"), torch.zeros(1, heads, device="cuda")
    pools = [x.view(pages, 1, page, 48).cuda().expand(-1, heads, -1, -1) for x in (keys, values)]
    ibp.ibp_attn_decode4(q.cuda().expand(1, heads, dim), *pools, torch.arange(pages, dtype=torch.int32, device="cuda")[None], int32([n]), n, out,
                         lse, scale=1.0)
    assert torch.equal(out, out[:, :1].expand_as(out)) and torch.equal(lse, lse[:, :1].expand_as(lse))
    near(q[0, 0], keys[:n], values[:n], out[0, 0].cpu(), lse[0, 0].cpu())
