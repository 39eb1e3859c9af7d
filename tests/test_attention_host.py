"""The attention entry points' checks of arguments (no GPU needed): every call that is refused
returns before anything is enqueued, with a status and a message."""
import ctypes
import os
import subprocess
import sys

import pytest

import paper_2605_30728_amd as ibp

torch = pytest.importorskip("torch")
ibp.ibp_attn_prompt                                   # (loads the signatures)
from paper_2605_30728_amd import attention as at      # noqa: E402

A = 1 << 20                                           # an aligned address that no refused call follows


def attn(**x):
    return at.ibp_attn(*({**dict(type=0, q_heads=4, kv_heads=2, head_dim=64, scale=0.125, flags=0), **x}.values()))


def rows(n=8, heads=4, **x):
    return at.ibp_rows(*({**dict(data=A, rows=n, row_stride=heads * 64, head_stride=64), **x}.values()))


def pages(**x):
    base = dict(keys=A, values=A, n_pages=4, page_tokens=16, table_pages=2, d_table=A, kp=2048, kh=1024, kt=64, vp=2048, vh=1024, vt=64)
    return at.ibp_pages(*({**base, **x}.values()))


def status(f, *args):
    s = getattr(ibp.lib(), f)(*args)
    assert s == ibp.IBP_OK or ibp.ibp_last_error() != ""
    return s


def prompt(a=None, q=None, k=None, v=None, qs=A, ks=A, n=1, out=None):
    return status("ibp_attn_prompt", a or attn(), q or rows(), k or rows(heads=2), v or rows(heads=2), qs, ks, n, out or rows(), A, A, 1 << 30, None)


BAD_ATTN = [dict(type=2), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=5), dict(q_heads=65538), dict(head_dim=0), dict(head_dim=4),
            dict(head_dim=12), dict(head_dim=264), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
            dict(scale=float("nan")), dict(scale=1e-38), dict(flags=2)]
BAD_ROWS = [dict(data=None), dict(data=A + 8), dict(row_stride=12), dict(head_stride=4), dict(row_stride=(1 << 23) + 8),
            dict(head_stride=(1 << 40) + 8), dict(n=1 << 31)]
BAD_PAGES = [dict(page_tokens=0), dict(page_tokens=(1 << 24) + 1), dict(n_pages=1 << 31), dict(keys=None), dict(values=None),
             dict(keys=A + 8), dict(d_table=None), dict(d_table=A + 2), dict(kp=2044), dict(vt=60), dict(vh=(1 << 40) + 8)]


def name(x):
    return ",".join(f"{k}={v}" for k, v in x.items())


@pytest.mark.parametrize("bad", BAD_ATTN, ids=name)
def test_parameters_are_checked(bad):
    a = attn(**bad)
    assert prompt(a=a) == ibp.IBP_EINVAL
    assert status("ibp_attn_key_weights", a, rows(), rows(heads=2), A, A, 1, A, A, A, 1 << 20, None) == ibp.IBP_EINVAL
    assert status("ibp_attn_decode", a, rows(), pages(), A, 20, rows(), None, None, 0, A, 1 << 30, None) == ibp.IBP_EINVAL
    assert status("ibp_kv_evict", a, pages(), A, 1, 20, 5, 1, A, A, A, 20, A, A, 20, A, A, 1 << 30, None) == ibp.IBP_EINVAL


@pytest.mark.parametrize("bad", BAD_ROWS, ids=name)
def test_rows_are_checked(bad):
    for which in ("q", "k", "v", "out"):
        assert prompt(**{which: rows(heads=4 if which in ("q", "out") else 2, **bad)}) == ibp.IBP_EINVAL
    assert status("ibp_attn_decode", attn(), rows(**bad), pages(), A, 20, rows(), None, None, 0, A, 1 << 30, None) == ibp.IBP_EINVAL


@pytest.mark.parametrize("bad", BAD_PAGES, ids=name)
def test_pages_are_checked(bad):
    assert status("ibp_attn_decode", attn(), rows(), pages(**bad), A, 20, rows(), None, None, 0, A, 1 << 30, None) == ibp.IBP_EINVAL
    assert status("ibp_kv_evict", attn(), pages(**bad), A, 1, 20, 5, 1, A, A, A, 20, A, A, 20, A, A, 1 << 30, None) == ibp.IBP_EINVAL


def test_prompt_refuses():
    L = ibp.lib()
    assert L.ibp_attn_prompt(None, rows(), rows(heads=2), rows(heads=2), A, A, 1, rows(), A, A, 0, None) == ibp.IBP_EINVAL
    assert L.ibp_attn_prompt(attn(), None, rows(heads=2), rows(heads=2), A, A, 1, rows(), A, A, 0, None) == ibp.IBP_EINVAL
    need = ctypes.c_uint64(0)
    assert status("ibp_attn_prompt_workspace", 4, 64, 8, 4096, 1, need) == ibp.IBP_OK and need.value > 0
    many = rows(4096, heads=2)
    assert L.ibp_attn_prompt(attn(), rows(), many, many, A, A, 1, rows(), A, A, need.value - 1, None) == ibp.IBP_ENOMEM
    assert L.ibp_attn_prompt(attn(), rows(), many, many, A, A, 1, rows(), A, None, 0, None) == ibp.IBP_EINVAL
    assert status("ibp_attn_prompt_workspace", 4, 64, 4096, 4096, 100, need) == ibp.IBP_OK and need.value == 0
    assert status("ibp_attn_prompt_workspace", 0, 64, 8, 8, 1, need) == ibp.IBP_EINVAL
    assert status("ibp_attn_prompt_workspace", 4, 12, 8, 8, 1, need) == ibp.IBP_EINVAL
    assert status("ibp_attn_prompt_workspace", 4, 64, 8, 8, 1, None) == ibp.IBP_EINVAL
    assert prompt(qs=None) == ibp.IBP_EINVAL and prompt(ks=None) == ibp.IBP_EINVAL and prompt(qs=A + 1) == ibp.IBP_EINVAL
    assert prompt(n=(1 << 24) + 1) == ibp.IBP_EINVAL
    assert prompt(v=rows(7, heads=2)) == ibp.IBP_EINVAL
    assert prompt(out=rows(7)) == ibp.IBP_ENOMEM
    assert prompt(q=rows(1 << 30), out=rows(1 << 30)) == ibp.IBP_EINVAL          # more blocks than a launch has
    assert prompt(n=0) == ibp.IBP_OK and prompt(q=rows(0), out=rows(0)) == ibp.IBP_OK     # nothing to do


def test_key_weights_refuse():
    call = lambda **x: status("ibp_attn_key_weights", *({**dict(a=attn(), q=rows(), k=rows(heads=2), qs=A, ks=A, n=1, lse=A, w=A, s=A,  # noqa: E731
                                                              sb=1 << 20, stream=None), **x}.values()))
    assert call(lse=None) == ibp.IBP_EINVAL and call(w=None) == ibp.IBP_EINVAL and call(s=None) == ibp.IBP_EINVAL
    assert call(s=A + 4) == ibp.IBP_EINVAL
    need = ctypes.c_uint64(0)
    assert status("ibp_attn_key_weights_workspace", 4, 2, 8, 1, need) == ibp.IBP_OK and need.value > 0
    assert call(sb=need.value - 1) == ibp.IBP_ENOMEM
    most = need.value
    for n in (2, 7, 31, 32, 1000):
        assert status("ibp_attn_key_weights_workspace", 4, 2, 8, n, need) == ibp.IBP_OK and need.value <= most
    assert status("ibp_attn_key_weights_workspace", 4, 4, 8, 32, need) == ibp.IBP_OK and need.value == 0
    assert status("ibp_attn_key_weights_workspace", 4, 3, 8, 1, need) == ibp.IBP_EINVAL
    assert status("ibp_attn_key_weights_workspace", 4, 2, 8, 1, None) == ibp.IBP_EINVAL


def test_decode_refuses():
    base = dict(a=attn(), q=rows(), g=pages(), lens=A, max_len=20, out=rows(), lse=None, w=None, ws=0, s=A, sb=1 << 30, stream=None)
    call = lambda **x: status("ibp_attn_decode", *({**base, **x}.values()))  # noqa: E731
    assert call(a=attn(flags=1)) == ibp.IBP_EINVAL
    assert call(g=None) == ibp.IBP_EINVAL and call(lens=None) == ibp.IBP_EINVAL
    assert call(max_len=33) == ibp.IBP_ERANGE and call(out=rows(7)) == ibp.IBP_ENOMEM
    assert call(w=A, ws=19) == ibp.IBP_ENOMEM
    need = ctypes.c_uint64(0)
    assert status("ibp_attn_decode_workspace", 8, 4, 2, 64, 20, 1, need) == ibp.IBP_OK and need.value > 0
    assert call(w=A, ws=20, sb=need.value - 1) == ibp.IBP_ENOMEM and call(w=A, ws=20, s=None) == ibp.IBP_EINVAL
    assert call(q=rows(0), out=rows(0), w=A, ws=20) == ibp.IBP_OK
    for bad in ((8, 4, 3, 64, 20, 0), (8, 4, 2, 60, 20, 0), (8, 4, 2, 64, 0x7fffffff, 0), (8, 4, 2, 264, 20, 0)):
        assert status("ibp_attn_decode_workspace", *bad, need) == ibp.IBP_EINVAL
    assert status("ibp_attn_decode_workspace", 8, 4, 2, 64, 20, 1, None) == ibp.IBP_EINVAL


def test_evict_refuses():
    base = dict(a=attn(), g=pages(), lens=A, n=1, max_len=20, budget=5, recent=1, nxt=A, w=A, p=A, stride=20, nw=A + 4096, np=A + 4096,
                ns=20, nl=A, s=A, sb=1 << 30, stream=None)
    call = lambda **x: status("ibp_kv_evict", *({**base, **x}.values()))  # noqa: E731
    for null in ("g", "lens", "nxt", "w", "p", "nw", "np", "nl", "s"):
        assert call(**{null: None}) == ibp.IBP_EINVAL
    assert call(budget=0) == ibp.IBP_EINVAL and call(recent=6) == ibp.IBP_EINVAL and call(max_len=33) == ibp.IBP_ERANGE
    assert call(stride=19) == ibp.IBP_EINVAL and call(ns=4) == ibp.IBP_ENOMEM
    assert call(nw=A, ns=19) == ibp.IBP_EINVAL                    # in place with another stride
    need = ctypes.c_uint64(0)
    assert status("ibp_kv_evict_workspace", 1, 2, 20, 5, need) == ibp.IBP_OK and need.value > 0
    assert call(sb=need.value - 1) == ibp.IBP_ENOMEM
    assert call(n=0) == ibp.IBP_OK
    assert status("ibp_kv_evict_workspace", 1, 0, 20, 5, need) == ibp.IBP_EINVAL
    assert status("ibp_kv_evict_workspace", 1, 2, 20, 0, need) == ibp.IBP_EINVAL


def test_evict_takes_no_more_slots_than_it_counts():
    """A block's threads go a round beyond the last slot, and a list of moves has two numbers for each: both have
    to fit 31 bits."""
    most, need = (1 << 31) - (1 << 24), ctypes.c_uint64(0)
    assert status("ibp_kv_evict_workspace", 1, 2, most, 5, need) == ibp.IBP_OK
    for beyond in (most + 1, (1 << 31) - 256):
        assert status("ibp_kv_evict_workspace", 1, 2, beyond, 5, need) == ibp.IBP_EINVAL
        g = pages(page_tokens=1 << 24, table_pages=128)
        assert status("ibp_kv_evict", attn(), g, A, 1, beyond, 5, 1, A, A, A, beyond, A + 4096, A + 4096, 20, A, A, 1 << 30, None) == ibp.IBP_EINVAL


def growing(call, sizes):
    """Whether the workspace call's answers never fall along the sizes."""
    need = [call(*x) for x in sizes]
    return all(a <= b for a, b in zip(need, need[1:]))


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim", [(32, 8, 128), (8, 1, 256), (6, 2, 64), (16, 16, 80), (600, 600, 8), (64, 1, 128)])
def test_decode_workspace_is_enough_for_smaller_calls(heads, kv_heads, dim, weights):
    """A program takes one workspace, of its most sequences and longest cache."""
    lens = sorted({128 * n + d for n in range(1, 140) for d in (-1, 0, 1)} | {1 << n for n in range(31)} | {3 << n for n in range(29)} | {0})
    call = lambda n, m: ibp.ibp_attn_decode_workspace(n, heads, kv_heads, dim, m, weights)  # noqa: E731
    for n in (1, 2, 3, 5, 24, 64):
        assert growing(call, [(n, m) for m in lens])
    for m in (100, 513, 5500, 8193, 131071):
        assert growing(call, [(n, m) for n in range(80)])


@pytest.mark.parametrize("heads,dim", [(32, 128), (16, 64), (1, 256), (5, 80), (40, 128), (200, 8), (600, 64)])
def test_prompt_workspace_is_enough_for_smaller_calls(heads, dim):
    """Of fewer rows of queries or keys, or more sequences that they belong to: few rows are split more than many."""
    rows = sorted({128 * n + d for n in range(1, 70) for d in (-1, 0, 1)} | {1, 8, 77, 8192, 20001, 1 << 20} | {0})
    call = lambda q, k, n: ibp.ibp_attn_prompt_workspace(heads, dim, q, k, n)  # noqa: E731
    for n in (1, 2, 3, 11):
        for k in (512, 1024, 5000, 9001, 131072):
            assert growing(call, [(q, k, n) for q in rows])
        for q in (1, 128, 1000, 8192):
            assert growing(call, [(q, k, n) for k in sorted({512 * n for n in range(20)} | {512 * n - 1 for n in range(1, 20)} | {1 << 20})])
    for q in (1, 300, 4096):
        assert growing(call, [(q, 9001, n) for n in range(20, 0, -1)])


def test_binding_refuses_host_tensors():
    q, starts = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(TypeError):
        ibp.ibp_attn_prompt(q, q, q, starts, starts, q)
    with pytest.raises(TypeError):
        ibp.ibp_kv_evict(q[None], q[None], starts[None], starts[:1], 4, 2, 1, starts[:1], q, q, q, q, starts[:1])


@pytest.mark.parametrize("call,good", [("ibp_attn_prompt_workspace", (4, 64, 100, 200, 1)), ("ibp_attn_key_weights_workspace", (4, 2, 100, 1)),
                                       ("ibp_attn_decode_workspace", (2, 4, 2, 64, 300)), ("ibp_kv_evict_workspace", (2, 2, 300, 100))])
def test_counts_of_more_than_32_bits_are_refused(call, good):
    """Not taken as what their low 32 bits say."""
    more = (True,) if call == "ibp_attn_decode_workspace" else ()
    assert getattr(ibp, call)(*good, *more) >= 0
    for i, x in enumerate(good):
        for bad in (x + (1 << 32), -1):
            with pytest.raises(ValueError):
                getattr(ibp, call)(*good[:i], bad, *good[i + 1:], *more)


@pytest.mark.parametrize("first", ["from paper_2605_30728_amd.attention import ibp_attn_prompt_workspace as f",
                                   "import paper_2605_30728_amd as ibp; f = ibp.ibp_attn_prompt_workspace",
                                   "from paper_2605_30728_amd import attention, ibp_attn_prompt_workspace as f; assert f is attention.ibp_attn_prompt_workspace"])
def test_the_operators_are_reached_from_module_and_package(first):
    """In a program that has not asked the package for them before."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(ibp.__file__)))
    done = subprocess.run([sys.executable, "-c", f"{first}; print(f(4, 64, 8, 4096, 1) > 0)"], cwd=root, capture_output=True, text=True)
    assert (done.returncode, done.stdout.strip()) == (0, "True"), done.stderr
