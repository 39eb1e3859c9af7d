"""Reading 4-bit records back where what they stand for passes the type's largest number: a step is rounded, so that the ends
of a group that holds that number may lie beyond it."""
import pytest
import torch

from kv_reference import held_bound, record_bytes, records_of, values_of
from test_gpu_kv4 import int32

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ibp():
    import paper_2605_30728_amd
    return paper_2605_30728_amd


def read(ibp, records, kind, dim):
    """Rows of records [n][heads][bytes], as keys and as values of one sequence."""
    n, heads = records.shape[:2]
    pool = records.transpose(0, 1).unsqueeze(0).contiguous().cuda()
    k, v = (torch.full((n, heads, dim), 7.0, dtype=kind, device="cuda") for _ in range(2))
    ibp.ibp_kv4_read(pool, pool, int32([[0]]), int32([n]), k, v, int32([0, n]))
    assert torch.equal(k.view(torch.int16), v.view(torch.int16))
    return k.cpu()


def in_range(records, dim, kind):
    """What groups of finite step and centre stand for, rounded to 32 bits, held to the type's largest numbers; others as they are."""
    top, x = torch.finfo(kind).max, values_of(records, dim, kind).float()
    n = -(-dim // 32)
    meta = records[..., 16 * n:20 * n].contiguous().view(kind)
    held = (meta[..., :n].isfinite() & meta[..., n:].isfinite()).repeat_interleave(32, -1)[..., :dim]
    return torch.where(held, x.clamp(-top, top), x).to(kind)


@pytest.mark.parametrize("rows", [30, 3000])
@pytest.mark.parametrize("kind", [BF16, F16])
def test_the_largest_numbers_come_back(ibp, kind, rows):
    """Appended and read: finite, and no further off than a held value is, to the rounding of what is read."""
    dim, heads, top = 128, 2, torch.finfo(kind).max
    g = torch.Generator().manual_seed(1)
    x = (torch.rand(rows, heads, dim, generator=g) * 2 - 1) * top
    x[..., 0], x[..., 33], x[..., 64], x[..., 65] = top, -top, top, -top
    x[:, 1, 96:] = top
    x = x.to(kind)
    pools = [torch.zeros(1, heads, rows, record_bytes(dim), dtype=torch.uint8, device="cuda") for _ in range(2)]
    lens, starts = int32([rows]), int32([0, rows])
    ibp.ibp_kv4_append(x.cuda(), x.cuda(), *pools, int32([[0]]), lens, lens, starts)
    k, v = (torch.zeros_like(x, device="cuda") for _ in range(2))
    ibp.ibp_kv4_read(*pools, int32([[0]]), lens, k, v, starts)
    records = records_of(x.float(), kind)
    for pool, got in zip(pools, (k.cpu(), v.cpu())):
        assert torch.equal(pool[0].transpose(0, 1).cpu(), records)
        assert got.isfinite().all()
        assert torch.equal(got, in_range(records, dim, kind))
        assert ((got.double() - x.double()).abs() <= held_bound(x, records, kind) + torch.finfo(kind).eps / 2 * got.double().abs()).all()


@pytest.mark.parametrize("kind", [BF16, F16])
def test_steps_and_centres_of_every_size(ibp, kind):
    """Records of a program's own making: those of finite numbers read finite, others as not finite as before."""
    dim, n = 64, 400
    g = torch.Generator().manual_seed(2)
    records = torch.randint(0, 256, (n, 2, record_bytes(dim)), generator=g, dtype=torch.uint8)
    meta = torch.randint(-1 << 15, 1 << 15, (n, 2, 4), generator=g).to(torch.int16).view(kind).clone()
    meta[:60, :, :2], meta[60:80, :, 2:] = torch.finfo(kind).max, torch.finfo(kind).max
    meta[:20, :, 2:], meta[80, :, 0], meta[81, :, 2] = -torch.finfo(kind).max, float("inf"), float("-inf")
    records[..., 32:40] = meta.view(torch.uint8)
    got, want = read(ibp, records, kind, dim), in_range(records, dim, kind)
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(5.0, 6.0, 7.0), want.nan_to_num(5.0, 6.0, 7.0))
    assert want.isinf().any() and want.isnan().any() and (want.abs() == torch.finfo(kind).max).any()
