"""The serving example at small sizes: its rows are the stored ones, and every result that it computes on the
way is the definition's."""
import importlib.util
import os

import pytest
import torch

from attention_reference import attend, key_weights

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("kv_serving", os.path.join(HERE, "..", "examples", "kv_serving.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("history,turn,budget", [((45, 0, 70), (9, 5, 33), 48), ((0,), (1,), 4), ((130,), (2,), 400)])
def test_every_result(example, history, turn, budget):
    q_heads, kv_heads, dim, page, recent = 6, 2, 64, 16, 4
    group, scale = q_heads // kv_heads, dim ** -0.5
    tokens = []

    def on_token(q, cache, out, before):
        torch.cuda.synchronize()
        q, out, lens, table = q.cpu(), out.cpu(), cache.lens.tolist(), cache.table.cpu().long()
        pools, was, now = (cache.k.cpu(), cache.v.cpu()), before.cpu(), cache.weights.cpu()
        for b, n in enumerate(lens):
            assert n <= budget + 1
            positions = cache.positions[b, :, :n].cpu()
            for g in range(kv_heads):
                k, v = (x[table[b], g].reshape(-1, dim)[:n] for x in pools)
                total, total_tol = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
                assert len(set(positions[g].tolist())) == n            # no slot was lost or doubled
                assert positions[g].max() == int(cache.next[b]) - 1
                for h in range(g * group, (g + 1) * group):
                    seen = torch.ones(1, n, dtype=torch.bool)
                    want, lse, tol, lse_tol = attend(q[b, h:h + 1], k, v, scale, seen)
                    assert ((out[b, h].double() - want[0]).abs() <= tol[0]).all()
                    w, w_tol = key_weights(q[b, h:h + 1], k, lse.float(), scale, seen)
                    total += w
                    total_tol += w_tol + w * (lse_tol + 2.0 ** -24 * lse.abs())
                bound = total_tol + 2.0 ** -23 * (was[b, g, :n].double() + total) * (group + 1)
                assert ((now[b, g, :n].double() - was[b, g, :n].double() - total).abs() <= bound).all()
        tokens.append(lens)

    prompt, cache, _ = example.run(history, turn, 5, q_heads, kv_heads, dim, budget, recent, page, seed=3, on_token=on_token)
    stored = example.rows_of(history, kv_heads, dim, 3)
    q, k, v, out, lse, weights = (prompt[x].cpu() for x in ("q", "k", "v", "out", "lse", "weights"))
    start = 0
    for b, (n, t) in enumerate(zip(history, turn)):
        q0, k0, m = int(prompt["q_starts"][b]), int(prompt["k_starts"][b]), n + t
        for x, rows in enumerate((k, v)):
            assert torch.equal(rows[k0:k0 + n], stored[x, :, start:start + n].transpose(0, 1))
        start += n
        seen = torch.arange(m)[None, :] <= torch.arange(t)[:, None] + n
        for g in range(kv_heads):
            total, total_tol = torch.zeros(m, dtype=torch.float64), torch.zeros(m, dtype=torch.float64)
            for h in range(g * group, (g + 1) * group):
                want, want_lse, tol, lse_tol = attend(q[q0:q0 + t, h], k[k0:k0 + m, g], v[k0:k0 + m, g], scale, seen)
                assert ((out[q0:q0 + t, h].double() - want).abs() <= tol).all()
                assert ((lse[h, q0:q0 + t].double() - want_lse).abs() <= lse_tol).all()
                w, w_tol = key_weights(q[q0:q0 + t, h], k[k0:k0 + m, g], lse[h, q0:q0 + t], scale, seen)
                total, total_tol = total + w, total_tol + w_tol
            assert ((weights[g, k0:k0 + m].double() - total).abs() <= total_tol + 2.0 ** -23 * group * total).all()
    assert len(tokens) == 5 and cache.next.tolist() == [n + t + 5 for n, t in zip(history, turn)]
    assert cache.lens.tolist() == [min(n + t + 5, budget) for n, t in zip(history, turn)]


def test_one_workspace_serves_a_cache_at_its_budget(example):
    """The loop's decode workspace is that of the whole cache, its calls are shorter: 5,401 slots of 5,500, between
    which the number of splits falls."""
    tokens = []
    _, cache, _ = example.run((5400, 0, 0), (100, 1, 1), 2, 32, 8, 128, 5400, 64, 32,
                              on_token=lambda q, cache, out, before: tokens.append((cache.lens.tolist(), bool(torch.isfinite(out.float()).all()))))
    assert tokens == [([5401, 2, 2], True), ([5401, 3, 3], True)]
    assert cache.lens.tolist() == [5400, 3, 3] and cache.next.tolist() == [5502, 3, 3]
