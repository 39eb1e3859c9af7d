"""Attention over prompts and the keys' weights against their definition in 64 bits."""
import pytest
import torch

from attention_reference import UNIT, attend, key_weights, visible

pytestmark = pytest.mark.gpu
NEG = float("-inf")
BF16, F16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ibp():
    import paper_2605_30728_amd
    return paper_2605_30728_amd


def starts(lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32)


def inputs(kind, heads, kv_heads, dim, q_lens, k_lens, seed=0, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    new = lambda n, h: torch.randn(n, h, dim, generator=g).mul_(gain).to(kind)  # noqa: E731
    return new(sum(q_lens), heads), new(sum(k_lens), kv_heads), new(sum(k_lens), kv_heads)


def run_prompt(ibp, q, k, v, q_lens, k_lens, causal=True, scale=None, out=None):
    dq, dk, dv = (x if x.is_cuda else x.cuda() for x in (q, k, v))
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda") if out is None else out
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device="cuda")
    ibp.ibp_attn_prompt(dq, dk, dv, starts(q_lens).cuda(), starts(k_lens).cuda(), out, lse, causal=causal, scale=scale)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu()


def check_prompt(q, k, v, q_lens, k_lens, out, lse, causal=True, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    group = q.shape[1] // k.shape[1]
    q0 = k0 = 0
    for ql, kl in zip(q_lens, k_lens):
        rq, rk = slice(q0, q0 + ql), slice(k0, k0 + kl)
        q0, k0 = q0 + ql, k0 + kl
        for h in range(q.shape[1]):
            o, x, o_tol, x_tol = attend(q[rq, h], k[rk, h // group], v[rk, h // group], scale, visible(ql, kl, causal))
            none = x == NEG
            assert torch.equal(lse[h, rq] == NEG, none)
            assert (out[rq, h][none] == 0).all()
            assert ((lse[h, rq][~none].double() - x[~none]).abs() <= x_tol[~none]).all()
            off = (out[rq, h].double() - o).abs()
            assert torch.isfinite(out[rq, h]).all() and (off <= o_tol).all(), (h, (off / o_tol.clamp(min=1e-30)).max())


LENGTHS = [([1], [1]), ([33], [33]), ([129, 0, 1, 64, 200], [129, 0, 1, 64, 200]), ([5, 1, 70], [300, 65, 70]),
           ([40, 130, 3], [7, 100, 0]), ([2], [1500])]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", LENGTHS, ids=[f"q{a}-k{b}".replace(" ", "") for a, b in LENGTHS])
@pytest.mark.parametrize("kind,heads,kv_heads,dim", [(BF16, 4, 2, 128), (F16, 3, 1, 64), (BF16, 2, 2, 80), (F16, 2, 1, 256)])
def test_prompt(ibp, kind, heads, kv_heads, dim, lens, causal):
    q, k, v = inputs(kind, heads, kv_heads, dim, *lens)
    out, lse = run_prompt(ibp, q, k, v, *lens, causal=causal)
    check_prompt(q, k, v, *lens, out, lse, causal=causal)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("dim", [8, 24, 40, 72, 96, 104, 136, 192, 248])
def test_prompt_head_dims(ibp, kind, dim):
    lens = [97, 31], [97, 140]
    q, k, v = inputs(kind, 2, 1, dim, *lens, seed=dim)
    out, lse = run_prompt(ibp, q, k, v, *lens)
    check_prompt(q, k, v, *lens, out, lse)


@pytest.mark.parametrize("heads,kv_heads", [(8, 8), (16, 8), (12, 4), (5, 1), (16, 16), (40, 8)])
def test_prompt_head_groups(ibp, heads, kv_heads):
    lens = [150, 20], [150, 20]
    q, k, v = inputs(BF16, heads, kv_heads, 64, *lens, seed=heads)
    out, lse = run_prompt(ibp, q, k, v, *lens)
    check_prompt(q, k, v, *lens, out, lse)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("scale", [0.01, 1.0, 30.0])
def test_prompt_scales_and_moving_maximum(ibp, kind, scale):
    """Keys whose scores grow along the sequence, so that the running reference moves in every tile, and
    scales from nearly uniform weights to one key taking all."""
    lens = [64], [700]
    q, k, v = inputs(kind, 2, 1, 64, *lens, seed=3)
    k = (k.float() * torch.linspace(0.01, 2.0, 700)[:, None, None]).to(kind)
    out, lse = run_prompt(ibp, q, k, v, *lens, scale=scale)
    check_prompt(q, k, v, *lens, out, lse, scale=scale)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,heads,kv_heads,dim", [(BF16, 8, 8, 64), (F16, 2, 1, 80), (BF16, 3, 1, 128), (F16, 1, 1, 256)])
def test_prompt_few_rows_many_keys(ibp, kind, heads, kv_heads, dim, causal):
    """Split along the keys and joined; a sequence too short for its share of the splits beside a long one, and
    a NaN and an infinity that the last rows see."""
    lens = [40, 1, 130], [3100, 9, 2000]
    assert ibp.ibp_attn_prompt_workspace(heads, dim, 171, 5109, 3) > 0
    q, k, v = inputs(kind, heads, kv_heads, dim, *lens, seed=dim)
    out, lse = run_prompt(ibp, q, k, v, *lens, causal=causal)
    check_prompt(q, k, v, *lens, out, lse, causal=causal)
    if causal:
        clean = v.clone()
        v[3099, 0, 1], v[5106, 0, 2] = float("inf"), float("nan")     # seen by row 39, and by rows 168 on
        bad, bad_lse = run_prompt(ibp, q, k, v, *lens)
        check_prompt(q, k, clean, *lens, out, bad_lse)                # (values have no part in an lse)
        first = slice(0, heads // kv_heads)
        assert (bad[39, first, 1].float() == float("inf")).all() and torch.isnan(bad[168:, first, 2]).all()
        bad[39, first, 1], bad[168:, first, 2] = out[39, first, 1], out[168:, first, 2]
        assert torch.isfinite(bad).all()
        assert torch.allclose(bad.float(), out.float(), rtol=0.02, atol=0.02)


@pytest.mark.parametrize("kind", [F16, BF16])
@pytest.mark.parametrize("heads,dim,rows,n", [(1, 64, 3, 6000), (1, 128, 2, 300), (600, 64, 2, 9000), (300, 128, 1, 20000), (300, 256, 2, 6000)])
def test_prompt_one_key_above_many(ibp, kind, heads, dim, rows, n):
    """One key takes nearly all of the weight and has a value of 0; what the others, at 2^-25 to 2^-30 of its weight,
    add up to is the output. None of them may be lost, with the keys split (few heads) or not: `attend`'s bound, with
    float16's spacing taken at the 2^12 by which its weights are lifted before they are rounded."""
    g = torch.Generator().manual_seed(n)
    q, k = torch.zeros(rows, 1, dim, dtype=kind), torch.randn(n, 1, dim, generator=g).to(kind)
    k[:, 0, 0] = -(17.5 + 3.5 * torch.rand(n, generator=g)).to(kind)     # (the rest is not seen by q)
    q[:, 0, 0] = 1.0
    v = (0.5 + torch.rand(n, 1, dim, generator=g)).to(kind)
    k[n // 3, 0, 0], v[n // 3] = 0.0, 0.0
    out, lse = run_prompt(ibp, q.expand(rows, heads, dim).cuda(), k.cuda(), v.cuda(), [rows], [n], scale=1.0)
    assert torch.equal(out, out[:, :1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
    o, x, o_tol, x_tol = attend(q[:, 0], k[:, 0], v[:, 0], 1.0, visible(rows, n, True))
    if kind == F16:
        o_tol -= 2.0 ** -24 * (1 - 2.0 ** -12) * v[:n - rows + 1, 0].double().sum(0)     # (at least these are seen)
    assert ((lse[0].double() - x).abs() <= x_tol).all()
    off = (out[:, 0].double() - o).abs()
    assert (off <= o_tol).all(), (off / o).max()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("falling", [False, True])
@pytest.mark.parametrize("kind", [F16, BF16])
def test_prompt_scores_of_millions(ibp, kind, falling, causal):
    """Scores from 0 to 6.5 million in steps of thousands: the largest that a row sees takes all, whatever the
    reference was before."""
    n = 1024
    q, k, v = inputs(kind, 1, 1, 64, [n], [n], seed=37)
    scores = torch.arange(n, dtype=torch.float32) * 64
    q[:] = 0
    q[:, 0, 0] = 1.0
    k[:, 0, 0] = (scores.flip(0) if falling else scores).to(kind)
    out, lse = run_prompt(ibp, q, k, v, [n], [n], causal=causal, scale=100.0)
    for i in range(0, n, 31):
        seen = k[:i + 1 if causal else n, 0, 0]
        top = seen.max()
        best = (seen == top).nonzero()[:, 0]                             # (bfloat16 has several of the largest)
        want, tol = v[best, 0].double().mean(0), 2.0 ** (-10 if kind == F16 else -7)
        assert ((out[i, 0].double() - want).abs() <= tol * v[best, 0].double().abs().mean(0) + 2.0 ** -24).all()
        assert abs(lse[0, i].item() - top.item() * 100.0) <= 2.0 ** -21 * top.item() * 100.0 + len(best)


def one_takes_all(q, k, v, scale, seen):
    """Per row: the value of the key with the highest score and that score, where it is so far above the next that the
    rest weighs nothing and no rounding of a score matters; None elsewhere."""
    rows = []
    for i in range(q.shape[0]):
        at = seen[i].nonzero()[:, 0]
        s = k[at].double() @ q[i].double()
        two = s.topk(min(2, len(at))).values
        rounding = (k[at].double().abs() @ q[i].double().abs()).max() * q.shape[1] * 2.0 ** -22
        clear = len(at) == 1 or ((two[0] - two[1]) * scale > 200 and two[0] - two[1] > rounding)
        rows.append((v[at[s.argmax()]], two[0].item() * scale) if len(at) and clear else None)
    return rows


@pytest.mark.parametrize("scale", [1e7, 1e9, 1e20, 1e30])
@pytest.mark.parametrize("lens", [([70], [300]), ([1], [1]), ([40, 3], [3100, 2000])], ids=["many", "one", "split"])
@pytest.mark.parametrize("kind", [BF16, F16])
def test_prompt_largest_scales(ibp, kind, lens, scale):
    """Scores of any size that 32 bits hold: one key takes all."""
    q, k, v = inputs(kind, 2, 1, 64, *lens, seed=43)
    out, lse = run_prompt(ibp, q, k, v, *lens, scale=scale)
    q0 = k0 = checked = 0
    for ql, kl in zip(*lens):
        for h in range(2):
            want = one_takes_all(q[q0:q0 + ql, h], k[k0:k0 + kl, 0], v[k0:k0 + kl, 0], scale, visible(ql, kl, True))
            for i, x in enumerate(want):
                if x is not None:
                    off = (out[q0 + i, h].double() - x[0].double()).abs()
                    assert (off <= 2.02 * UNIT[kind] * x[0].double().abs() + 2.0 ** -24).all()     # its weight's rounding, and its own
                    assert abs(lse[h, q0 + i].item() - x[1]) <= 2.0 ** -16 * abs(x[1])       # (a score's rounding, 64 products)
                    checked += 1
        q0, k0 = q0 + ql, k0 + kl
    assert checked > sum(lens[0])                                        # of 2 heads


def test_prompt_with_one_workspace_for_all_sizes(ibp):
    """The workspace of the most rows and keys, as one sequence, serves every call of fewer, with the result that a
    workspace of its own gives; what was refused before are the sizes that are split, after one that is not."""
    heads, dim, most = 16, 64, (3000, 6000)
    q, k, v = (x.cuda() for x in inputs(BF16, heads, 1, dim, [most[0]], [most[1]], seed=31))
    space = torch.empty(ibp.ibp_attn_prompt_workspace(heads, dim, *most, 1), dtype=torch.uint8, device="cuda")
    for q_lens, k_lens in ([3000], [6000]), ([1023], [6000]), ([1024], [6000]), ([77], [5000]), ([1], [1024]), ([500, 1, 300], [3000, 2, 2800]):
        nq, nk = sum(q_lens), sum(k_lens)
        results = []
        for w in (space, None):
            out, lse = torch.zeros_like(q[:nq]), torch.zeros(heads, nq, device="cuda")
            ibp.ibp_attn_prompt(q[:nq], k[:nk], v[:nk], starts(q_lens).cuda(), starts(k_lens).cuda(), out, lse, workspace=w)
            results.append((out, lse))
        assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
        if nq <= 100:
            check_prompt(q[:nq].cpu(), k[:nk].cpu(), v[:nk].cpu(), q_lens, k_lens, results[0][0].cpu(), results[0][1].cpu())


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompt_many_sequences(ibp, dim):
    """More sequences than a wave has lanes, empty ones among them."""
    q_lens = [(7 * i) % 13 for i in range(150)]
    k_lens = [n + (i % 3) for i, n in enumerate(q_lens)]
    q, k, v = inputs(BF16, 2, 2, dim, q_lens, k_lens, seed=5)
    out, lse = run_prompt(ibp, q, k, v, q_lens, k_lens)
    check_prompt(q, k, v, q_lens, k_lens, out, lse)


@pytest.mark.parametrize("kind", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 80, 128, 256])
def test_what_is_not_seen_has_no_effect(ibp, kind, dim):
    """NaN and infinities in keys and values that a row does not see: later tokens, other sequences, and
    rows of no sequence. The rows that do see them are as they should be too."""
    lens = [90, 150], [90, 150]
    q, k, v = inputs(kind, 2, 1, dim, *lens, seed=7)
    clean, clean_lse = run_prompt(ibp, q, k, v, *lens)
    for place in (40, 89, 130, 239):                 # tokens of the first and second sequence
        for bad in (float("nan"), float("inf"), float("-inf")):
            k2, v2 = k.clone(), v.clone()
            v2[place, 0, 1] = bad
            k2[place, 0, 0] = float("nan") if bad != bad else k2[place, 0, 0]
            out, lse = run_prompt(ibp, q, k2, v2, *lens)
            first = 0 if place < 90 else 90
            last = 90 if place < 90 else 240
            unseen = torch.ones(240, dtype=torch.bool)
            unseen[place:last] = False
            assert torch.isfinite(out[unseen]).all() and torch.isfinite(lse[:, unseen]).all()
            assert torch.allclose(out[unseen].float(), clean[unseen].float(), rtol=0.02, atol=0.02)
            assert torch.allclose(lse[:, unseen], clean_lse[:, unseen], rtol=1e-5, atol=1e-5)
            assert first <= place < last
            if bad != bad:
                assert torch.isnan(out[place:last]).all() and torch.isnan(lse[:, place:last]).all()
            else:
                assert (out[place:last, :, 1].float() == bad).all()
                rest = torch.arange(dim) != 1
                assert torch.allclose(out[place:last][..., rest].float(), clean[place:last][..., rest].float(), rtol=0.02, atol=0.02)


def test_scores_of_minus_infinity(ibp):
    """A key of -inf scores -inf for positive queries: no weight; a row with only such keys gives zeros."""
    q, k, v = inputs(BF16, 1, 1, 64, [70], [70], seed=1)
    q[:, :, 0] = 1.0
    k[:30, :, 0] = NEG
    out, lse = run_prompt(ibp, q, k, v, [70], [70])
    assert (lse[0, :30] == NEG).all() and (out[:30] == 0).all()
    keep_q, keep_k = q[30:], k[30:]
    o, x, o_tol, x_tol = attend(keep_q[:, 0], keep_k[:, 0], v[30:, 0], 64 ** -0.5, visible(40, 40, True))
    assert ((out[30:, 0].double() - o).abs() <= o_tol).all() and ((lse[0, 30:].double() - x).abs() <= x_tol).all()


@pytest.mark.parametrize("heads", [1, 300])
@pytest.mark.parametrize("sign", [1, -1])
def test_prompt_of_the_largest_values(ibp, heads, sign):
    """float16 values of 65504, as a program has that saturates them: so is their mean, whatever the rounding of the
    weights (of the later keys, each 2^-11 up) makes of it. Infinities stay what they are."""
    n = 4000
    q, k, v = (torch.zeros(r, 1, 64, dtype=F16) for r in (2, n, n))
    q[:, :, 0] = 1.0
    k[64:, :, 0] = 4.91e-4
    v[:] = sign * 65504.0
    v[n // 2, 0, 5] = sign * float("inf")
    out, lse = run_prompt(ibp, q.expand(2, heads, 64).cuda(), k.cuda(), v.cuda(), [2], [n], scale=1.0)
    rest = torch.arange(64) != 5
    assert (out[..., rest].float() == sign * 65504.0).all() and (out[..., 5].float() == sign * float("inf")).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("lens", [([70], [70]), ([40], [3100])], ids=["whole", "split"])
def test_rows_of_no_weight_give_zeros(ibp, lens, bad):
    """A row that sees only scores of -inf gives zeros, whatever the values are."""
    (n,), (m,) = lens
    q, k, v = inputs(F16, 1, 1, 64, *lens, seed=47)
    q[:, :, 0] = 1.0
    k[:m - n + 30, :, 0] = NEG
    at = m - n + 30                          # the keys from here on, which the rows from 30 on see as well
    _, x, _, x_tol = attend(q[30:, 0], k[at:, 0], v[at:, 0], 64 ** -0.5, visible(n - 30, n - 30, True))
    v[5, 0, 3], v[m - n + 10] = bad, bad
    out, lse = run_prompt(ibp, q, k, v, *lens)
    assert (out[:30] == 0).all() and (lse[0, :30] == NEG).all()
    assert ((lse[0, 30:].double() - x).abs() <= x_tol).all()


def test_prompt_strides(ibp):
    """Heads and rows in any order: slices of one fused tensor, [head][row] order, an output with gaps."""
    lens = [77, 60], [77, 60]
    q, k, v = inputs(BF16, 4, 2, 64, *lens, seed=9)
    want, want_lse = run_prompt(ibp, q, k, v, *lens)
    fused = torch.cat([q, k, v], 1).cuda()           # [row][q heads, k heads, v heads][dim]
    out = torch.full((137, 8, 72), 7.0, dtype=BF16, device="cuda")
    got, lse = run_prompt(ibp, fused[:, :4], fused[:, 4:6], fused[:, 6:], *lens, out=out[:, 1::2, :64])
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    assert (out[:, ::2] == 7).all() and (out[:, :, 64:] == 7).all()
    turned = [x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in (q, k, v)]
    got, lse = run_prompt(ibp, *turned, *lens)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    wide = torch.zeros(137, 2, 200, dtype=BF16, device="cuda")
    wide[..., 16:80] = k.cuda()
    got, _ = run_prompt(ibp, q, wide[..., 16:80], v, *lens)
    assert torch.equal(got, want)


def test_prompt_offsets_past_32_bits(ibp):
    """Rows so far apart that their byte offsets need more than 32 bits."""
    n, stride = 300, 1 << 23                         # 300 rows x 16 MiB
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(n, 1, 64, generator=g).to(BF16) for _ in range(3))
    pool = torch.empty((n - 1) * stride + 128, dtype=BF16, device="cuda")
    far = [torch.as_strided(pool, (n, 1, 64), (stride, 64, 1), 64 * i) for i in range(2)]
    far[0].copy_(k.cuda())
    far[1].copy_(v.cuda())
    want, want_lse = run_prompt(ibp, q, k, v, [n], [n])
    got, lse = run_prompt(ibp, q, far[0], far[1], [n], [n])
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    far[0].copy_(q.cuda())
    out, lse = run_prompt(ibp, far[0], k, v, [n], [n], out=far[1])
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_rows_of_no_sequence_are_left_alone(ibp):
    q, k, v = inputs(BF16, 2, 1, 64, [50], [50], seed=4)
    out = torch.full((50, 2, 64), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((2, 50), 7.0, device="cuda")
    at = torch.tensor([10, 30], dtype=torch.int32, device="cuda")
    ibp.ibp_attn_prompt(q.cuda(), k.cuda(), v.cuda(), at, at, out, lse)
    w = torch.full((1, 50), 7.0, device="cuda")
    ibp.ibp_attn_key_weights(q.cuda(), k.cuda(), at, at, lse, w)
    for x in (out.transpose(0, 1), lse, w):
        assert (x[:, :10] == 7).all() and (x[:, 30:] == 7).all() and (x[:, 10:30] != 7).any()
    check_prompt(q[10:30], k[10:30], v[10:30], [20], [20], out[10:30].cpu(), lse[:, 10:30].cpu())


def test_starts_out_of_range_are_clamped(ibp):
    """Starts are only read on the device: ones beyond the tensors end there, and a falling pair is empty."""
    q, k, v = inputs(BF16, 1, 1, 64, [40], [40], seed=4)
    want, want_lse = run_prompt(ibp, q, k, v, [40], [40])
    out = torch.full((40, 1, 64), 7.0, dtype=BF16, device="cuda")
    at = torch.tensor([-5, 400, 3], dtype=torch.int32, device="cuda")
    ibp.ibp_attn_prompt(q.cuda(), k.cuda(), v.cuda(), at, at, out)
    assert torch.equal(out.cpu(), want)


def test_empty_calls(ibp):
    none = torch.zeros(0, 2, 64, dtype=BF16, device="cuda")
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    ibp.ibp_attn_prompt(none, none, none, at, at, none)
    ibp.ibp_attn_key_weights(none, none, at, at, torch.zeros(2, 0, device="cuda"), torch.zeros(2, 0, device="cuda"))
    q = torch.ones(3, 2, 64, dtype=BF16, device="cuda")
    at, zero = torch.tensor([0, 3], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.zeros(2, 3, device="cuda")
    ibp.ibp_attn_prompt(q, none, none, at, zero, out, lse)
    assert (out == 0).all() and (lse == NEG).all()


def run_weights(ibp, q, k, q_lens, k_lens, lse, causal=True, scale=None):
    w = torch.full((k.shape[1], k.shape[0]), 7.0, device="cuda")
    ibp.ibp_attn_key_weights(q.cuda(), k.cuda(), starts(q_lens).cuda(), starts(k_lens).cuda(), lse.cuda(), w, causal=causal,
                             scale=scale)
    return w.cpu()


def check_weights(q, k, q_lens, k_lens, lse, w, causal=True, scale=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    group = q.shape[1] // k.shape[1]
    q0 = k0 = 0
    for ql, kl in zip(q_lens, k_lens):
        rq, rk = slice(q0, q0 + ql), slice(k0, k0 + kl)
        q0, k0 = q0 + ql, k0 + kl
        for g in range(k.shape[1]):
            parts = [key_weights(q[rq, h], k[rk, g], lse[h, rq], scale, visible(ql, kl, causal))
                     for h in range(g * group, (g + 1) * group)]
            want, tol = sum(p[0] for p in parts), sum(p[1] for p in parts)
            tol = tol + group * 2.0 ** -24 * want
            assert ((w[g, rk].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens", LENGTHS, ids=[f"q{a}-k{b}".replace(" ", "") for a, b in LENGTHS])
@pytest.mark.parametrize("kind,heads,kv_heads,dim", [(BF16, 4, 2, 128), (F16, 3, 1, 64), (BF16, 2, 2, 80), (F16, 2, 1, 256)])
def test_key_weights(ibp, kind, heads, kv_heads, dim, lens, causal):
    q, k, v = inputs(kind, heads, kv_heads, dim, *lens, seed=11)
    _, lse = run_prompt(ibp, q, k, v, *lens, causal=causal)
    w = run_weights(ibp, q, k, *lens, lse, causal=causal)
    check_weights(q, k, *lens, lse, w, causal=causal)


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 8, 40), (16, 2, 96), (7, 7, 136)])
def test_key_weights_heads_and_dims(ibp, heads, kv_heads, dim):
    lens = [70, 300], [70, 311]
    q, k, v = inputs(F16, heads, kv_heads, dim, *lens, seed=13)
    _, lse = run_prompt(ibp, q, k, v, *lens)
    check_weights(q, k, *lens, lse, run_weights(ibp, q, k, *lens, lse))


def test_key_weights_sum_to_the_rows(ibp):
    """Every row gives one in all: a sequence's weights sum to rows x query heads."""
    lens = [1000], [1000]
    q, k, v = inputs(BF16, 8, 2, 128, *lens, seed=17)
    _, lse = run_prompt(ibp, q, k, v, *lens)
    w = run_weights(ibp, q, k, *lens, lse)
    assert torch.allclose(w.double().sum(1), torch.full((2,), 4000.0, dtype=torch.float64), rtol=1e-5)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,heads,kv_heads,dim", [(BF16, 4, 2, 128), (F16, 3, 1, 64), (BF16, 1, 1, 96), (F16, 2, 1, 256)])
def test_key_weights_many_tiles_of_rows(ibp, kind, heads, kv_heads, dim, causal):
    """Blocks that stream many tiles of rows past their keys, several waves each loading a share of a tile: every
    tile counts once, the same every time."""
    lens = [2100], [300]
    q, k, v = inputs(kind, heads, kv_heads, dim, *lens, seed=29)
    _, lse = run_prompt(ibp, q, k, v, *lens, causal=causal)
    w = run_weights(ibp, q, k, *lens, lse, causal=causal)
    check_weights(q, k, *lens, lse, w, causal=causal)
    for _ in range(8):
        assert torch.equal(run_weights(ibp, q, k, *lens, lse, causal=causal), w)


def test_key_weights_ignore_what_does_not_count(ibp):
    """A NaN row counts only for the keys it sees, a NaN key only for itself, a row without an lse not at all."""
    lens = [150], [150]
    q, k, v = inputs(BF16, 2, 1, 128, *lens, seed=19)
    _, lse = run_prompt(ibp, q, k, v, *lens)
    clean = run_weights(ibp, q, k, *lens, lse)
    q2, lse2 = q.clone(), lse.clone()
    q2[60], lse2[:, 60] = float("nan"), float("nan")
    w = run_weights(ibp, q2, k, *lens, lse2)
    assert torch.isnan(w[:, :61]).all() and torch.equal(w[:, 61:], clean[:, 61:])
    k2 = k.clone()
    k2[90] = float("inf")
    w = run_weights(ibp, q, k2, *lens, lse)
    other = torch.arange(150) != 90
    assert torch.equal(w[:, other], clean[:, other])
    lse2 = lse.clone()
    lse2[:, 140] = NEG
    w = run_weights(ibp, q, k, *lens, lse2)
    check_weights(q, k, *lens, lse2, w)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), NEG])
@pytest.mark.parametrize("kind,dim", [(BF16, 128), (F16, 64)])
def test_key_weights_of_rows_without_an_lse(ibp, kind, dim, bad, causal):
    """A row of lse -inf gives nothing, whatever its query holds, and so whatever its scores are."""
    lens = [150, 70], [150, 70]
    q, k, v = inputs(kind, 2, 1, dim, *lens, seed=41)
    _, lse = run_prompt(ibp, q, k, v, *lens, causal=causal)
    rows = [0, 33, 64, 149, 150, 219]
    lse[:, rows] = NEG
    want = run_weights(ibp, q, k, *lens, lse, causal=causal)
    check_weights(q, k, *lens, lse, want, causal=causal)
    q[rows] = bad
    assert torch.equal(run_weights(ibp, q, k, *lens, lse, causal=causal), want)


def test_same_result_every_time_and_on_any_stream(ibp):
    lens = [300, 50], [300, 80]
    q, k, v = inputs(BF16, 8, 2, 128, *lens, seed=23)
    out, lse = run_prompt(ibp, q, k, v, *lens)
    w = run_weights(ibp, q, k, *lens, lse)
    for _ in range(3):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            again, again_lse = run_prompt(ibp, q, k, v, *lens)
            again_w = run_weights(ibp, q, k, *lens, lse)
        s.synchronize()
        assert torch.equal(again, out) and torch.equal(again_lse, lse) and torch.equal(again_w, w)


def test_binding_refuses(ibp):
    q, k, v = (x.cuda() for x in inputs(BF16, 2, 1, 64, [8], [8]))
    at = starts([8]).cuda()
    out, lse, w = torch.empty_like(q), torch.empty(2, 8, device="cuda"), torch.empty(1, 8, device="cuda")
    call = lambda **x: ibp.ibp_attn_prompt(*({**dict(q=q, k=k, v=v, a=at, b=at, out=out), **x}[n] for n in  # noqa: E731
                                             ("q", "k", "v", "a", "b", "out")), x.get("lse"), scale=x.get("scale"))
    for error, bad in [(TypeError, dict(q=q.cpu())), (TypeError, dict(q=q.float())), (TypeError, dict(k=k.half())),
                       (ValueError, dict(k=k[:, :, :56])), (ValueError, dict(v=v[0])), (TypeError, dict(a=at.long())),
                       (ValueError, dict(a=torch.cat([at, at]))), (ValueError, dict(lse=lse[:1])),
                       (TypeError, dict(out=out.cpu())), (ValueError, dict(out=out[:, :1])),
                       (TypeError, dict(q=q.transpose(1, 2).contiguous().transpose(1, 2))),
                       (ibp.IbpError, dict(scale=0.0)), (ibp.IbpError, dict(scale=float("nan"))),
                       (ibp.IbpError, dict(out=out[:4])), (ibp.IbpError, dict(v=v[:4]))]:
        with pytest.raises(error):
            call(**bad)
    with pytest.raises(ibp.IbpError) as e:           # 16-byte alignment
        shifted = torch.zeros(8 * 64 + 1, dtype=BF16, device="cuda")[1:].view(8, 1, 64)
        call(k=shifted)
    assert e.value.status == ibp.IBP_EINVAL
    with pytest.raises(ibp.IbpError) as e:
        ibp.ibp_attn_key_weights(q, k, at, at, lse, w, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == ibp.IBP_ENOMEM


@pytest.mark.parametrize("as_handle", [False, True])
def test_workspace_belongs_to_the_stream_of_the_call(ibp, as_handle):
    """A workspace that the call takes itself, on a stream that is still busy, is not handed to the program's
    current stream before the call's kernels are done with it."""
    q, k = (torch.randn(n, h, 64, device="cuda").bfloat16() for n, h in ((100, 4), (2000, 2)))
    starts = [torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (100, 2000)]
    lse, weights, want = torch.zeros(4, 100, device="cuda"), *(torch.zeros(2, 2000, device="cuda") for _ in range(2))
    need = ibp.ibp_attn_key_weights_workspace(4, 2, 2000, 1)
    ibp.ibp_attn_key_weights(q, k, *starts, lse, want)
    busy, side = torch.randn(4096, 4096, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(10):
            busy = busy @ busy * 1e-2
    ibp.ibp_attn_key_weights(q, k, *starts, lse, weights, stream=side.cuda_stream if as_handle else side)
    mine = torch.full((need,), 7, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert (mine == 7).all() and torch.equal(weights, want)


@pytest.mark.parametrize("which", ["null", "default", "handle", "current"])
def test_workspace_is_taken_on_the_stream_of_the_call(ibp, monkeypatch, which):
    """Whatever names the stream: the default one's handle is 0."""
    q, k = (torch.randn(n, h, 64, device="cuda").bfloat16() for n, h in ((100, 4), (2000, 2)))
    at = [torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (100, 2000)]
    lse, weights = torch.zeros(4, 100, device="cuda"), torch.zeros(2, 2000, device="cuda")
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    stream, handle = {"null": (0, 0), "default": (torch.cuda.default_stream(), 0), "handle": (other.cuda_stream, other.cuda_stream),
                      "current": (None, side.cuda_stream)}[which]
    torch.cuda.synchronize()
    taken, empty = [], torch.empty

    def recorded(*args, **kwargs):
        taken.append(torch.cuda.current_stream().cuda_stream)
        return empty(*args, **kwargs)

    with torch.cuda.stream(side):
        monkeypatch.setattr(torch, "empty", recorded)
        ibp.ibp_attn_key_weights(q, k, *at, lse, weights, stream=stream)
        monkeypatch.undo()
    torch.cuda.synchronize()
    assert taken == [handle]
