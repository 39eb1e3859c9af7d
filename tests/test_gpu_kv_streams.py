"""Appends to 4-bit caches and decodes over others at once, on streams and in workspaces of their own."""
import pytest
import torch

from kv_reference import record_bytes, rotation_table
from test_gpu_kv4 import Cache, decode, int32, queries

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def ibp():
    import paper_2605_30728_amd
    return paper_2605_30728_amd


def test_two_decodes_and_an_append_at_once(ibp):
    """Each leaves what it leaves alone, several times over."""
    c = [Cache(BF16, 2, 128, [3000, 500], 32, seed=s) for s in (19, 20)]
    q = [queries(x, 8, s).cuda() for s, x in enumerate(c)]
    caches = [(x.keys.cuda(), x.values.cuda(), x.table.cuda(), int32(x.lens)) for x in c]
    before = torch.rand(2, 2, 3000)
    want = [decode(ibp, x, y.cpu(), before) for x, y in zip(c, q)]
    need = ibp.ibp_attn_decode4_workspace(2, 8, 2, 128, 3000, True)
    spaces = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in c]
    outs = [(torch.zeros_like(y), torch.zeros(2, 8, device="cuda"), before.cuda()) for y in q]

    g = torch.Generator().manual_seed(21)
    rows, new, held = 700, [600, 100], [5, 40]
    k, v = (torch.randn(rows, 2, 128, generator=g).to(BF16).cuda() for _ in range(2))
    queries_in = torch.randn(rows, 8, 128, generator=g).to(BF16).cuda()
    lens, starts, table = int32([a + b for a, b in zip(new, held)]), int32([0, 600, 700]), torch.randperm(40, generator=g).view(2, 20).to(torch.int32).cuda()
    rotation = rotation_table(700, 64).cuda()

    def fresh():
        return [torch.full((40, 2, 32, record_bytes(128)), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2)], torch.zeros_like(queries_in)

    def append(pools, turned, stream=None):
        ibp.ibp_kv4_append(k, v, *pools, table, lens, lens, starts, rotation, q=queries_in, q_out=turned, stream=stream)

    alone, at_once = fresh(), fresh()
    append(*alone)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        for pool in at_once[0]:
            pool.fill_(0x5A)
        at_once[1].zero_()
        for out, lse, w in outs:
            out.zero_(), lse.zero_(), w.copy_(before)
        torch.cuda.synchronize()
        for x, y, space, s, (out, lse, w) in zip(caches, q, spaces, streams, outs):
            ibp.ibp_attn_decode4(y, *x, 3000, out, lse, weights=w, workspace=space, stream=s)
        append(*at_once, stream=streams[2])
        torch.cuda.synchronize()
        for got, expected in zip(outs, want):
            assert all(torch.equal(a.cpu(), b) for a, b in zip(got, expected))
        assert all(torch.equal(a, b) for a, b in zip((*at_once[0], at_once[1]), (*alone[0], alone[1])))
