"""Heads, head sizes and pairs beyond 32 bits, which the library's structures cannot hold: refused as values, not cut."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BIG = (1 << 32) + 8


def test_refusals():
    import paper_2605_30728_amd as ibp
    x = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    many = x[:, :1].expand(1, BIG, 64)
    pool, pool4 = torch.zeros(1, 1, 16, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 1, 16, 48, dtype=torch.uint8, device="cuda")
    one, table = torch.ones(1, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    turns = torch.zeros(0, 1 << 31, 2, device="cuda")
    for call, p in ((ibp.ibp_kv_append, pool), (ibp.ibp_kv4_append, pool4)):
        with pytest.raises(ValueError, match="fit 32 bits"):
            call(x, x, p, p, table, one, one, q=many, q_out=many)
        with pytest.raises(ValueError, match="fit 32 bits"):
            call(many, many, p.expand(1, BIG, *p.shape[2:]), p.expand(1, BIG, *p.shape[2:]), table, one, one)
        with pytest.raises(ValueError, match="fit 32 bits"):
            call(x, x, p, p, table, one, one, rotation=turns)
        call(x, x, p, p, table, one, one)
    with pytest.raises(ValueError, match="fit 32 bits"):
        ibp.ibp_kv4_read(*[pool4.expand(1, BIG, 16, 48)] * 2, table, one, many, many)
    with pytest.raises(ValueError, match="32 bits|2\\^32"):
        ibp.ibp_attn_decode4(many, pool4, pool4, table, one, 16, many)
