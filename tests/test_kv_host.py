"""The KV cache entry points' checks of arguments and the format of 4-bit records (no GPU needed)."""
import ctypes
import os
import subprocess
import sys

import pytest

import paper_2605_30728_amd as ibp

torch = pytest.importorskip("torch")
ibp.ibp_kv_append                                     # (loads the signatures)
from kv_reference import held_bound, record_bytes, records_of, values_of      # noqa: E402
from paper_2605_30728_amd import kv_cache as kc       # noqa: E402

A = 1 << 20                                           # an aligned address that no refused call follows


def attn(**x):
    return kc.ibp_attn(*({**dict(type=0, q_heads=4, kv_heads=2, head_dim=64, scale=1.0, flags=0), **x}.values()))


def rows(n=8, heads=2, **x):
    return kc.ibp_rows(*({**dict(data=A, rows=n, row_stride=heads * 64, head_stride=64), **x}.values()))


def pages(**x):
    base = dict(keys=A, values=A, n_pages=4, page_tokens=16, table_pages=2, d_table=A, kp=2048, kh=1024, kt=64, vp=2048, vh=1024, vt=64)
    return kc.ibp_pages(*({**base, **x}.values()))


def rotation(**x):
    return kc.ibp_rotation(*({**dict(d_table=A, positions=100, turned=64, halves=1), **x}.values()))


def status(f, *args):
    s = getattr(ibp.lib(), f)(*args)
    assert s == ibp.IBP_OK or ibp.ibp_last_error() != ""
    return s


def append(call="ibp_kv_append", **x):
    base = dict(a=attn(), k=rows(), v=rows(), q=rows(heads=4), q_out=rows(heads=4), r=rotation(), starts=A, n=1, g=pages(), lens=A, nxt=A, w=A,
                p=A, stride=20, stream=None)
    return status(call, *({**base, **x}.values()))


def read(**x):
    base = dict(a=attn(), g=pages(), lens=A, n=1, starts=A, first=A, k=rows(), v=rows(), stream=None)
    return status("ibp_kv4_read", *({**base, **x}.values()))


def decode(**x):
    base = dict(a=attn(), q=rows(heads=4), g=pages(), lens=A, max_len=20, out=rows(heads=4), lse=None, w=None, ws=0, s=A, sb=1 << 30, stream=None)
    return status("ibp_attn_decode4", *({**base, **x}.values()))


BAD_ATTN = [dict(type=2), dict(q_heads=0), dict(kv_heads=0), dict(q_heads=5), dict(q_heads=65538), dict(head_dim=0), dict(head_dim=12),
            dict(head_dim=264), dict(scale=0.0), dict(scale=float("nan")), dict(flags=2)]
BAD_ROWS = [dict(data=None), dict(data=A + 8), dict(row_stride=12), dict(head_stride=4), dict(row_stride=(1 << 23) + 8), dict(n=1 << 31)]
BAD_PAGES = [dict(page_tokens=0), dict(page_tokens=(1 << 24) + 1), dict(n_pages=1 << 31), dict(keys=None), dict(values=None),
             dict(keys=A + 8), dict(d_table=None), dict(d_table=A + 2), dict(kp=2044), dict(vt=60), dict(vh=(1 << 40) + 8)]


def name(x):
    return ",".join(f"{k}={v}" for k, v in x.items())


@pytest.mark.parametrize("bad", BAD_ATTN, ids=name)
def test_parameters_are_checked(bad):
    for call in ("ibp_kv_append", "ibp_kv4_append"):
        assert append(call, a=attn(**bad)) == ibp.IBP_EINVAL
    assert read(a=attn(**bad)) == ibp.IBP_EINVAL and decode(a=attn(**bad)) == ibp.IBP_EINVAL


@pytest.mark.parametrize("bad", BAD_ROWS, ids=name)
def test_rows_are_checked(bad):
    for call in ("ibp_kv_append", "ibp_kv4_append"):
        for which in ("k", "v", "q", "q_out"):
            assert append(call, **{which: rows(heads=4 if which[0] == "q" else 2, **bad)}) == ibp.IBP_EINVAL
    for which in ("k", "v"):
        assert read(**{which: rows(**bad)}) == ibp.IBP_EINVAL
    for which in ("q", "out"):
        assert decode(**{which: rows(heads=4, **bad)}) == ibp.IBP_EINVAL


@pytest.mark.parametrize("bad", BAD_PAGES, ids=name)
def test_pages_are_checked(bad):
    for call in ("ibp_kv_append", "ibp_kv4_append"):
        assert append(call, g=pages(**bad)) == ibp.IBP_EINVAL
    assert read(g=pages(**bad)) == ibp.IBP_EINVAL and decode(g=pages(**bad)) == ibp.IBP_EINVAL


@pytest.mark.parametrize("call", ["ibp_kv_append", "ibp_kv4_append"])
def test_append_refuses(call):
    for null in ("a", "k", "v", "q", "q_out", "g", "lens", "nxt"):
        assert append(call, **{null: None}) == ibp.IBP_EINVAL
    assert append(call, v=rows(7)) == ibp.IBP_EINVAL and append(call, q=rows(7, heads=4)) == ibp.IBP_EINVAL
    assert append(call, q_out=rows(7, heads=4)) == ibp.IBP_ENOMEM
    assert append(call, q_out=rows(heads=4, row_stride=512)) == ibp.IBP_EINVAL          # in place with another stride
    assert append(call, starts=A + 2) == ibp.IBP_EINVAL and append(call, n=(1 << 24) + 1) == ibp.IBP_EINVAL
    assert append(call, starts=None) == ibp.IBP_EINVAL                                  # eight rows of one sequence
    for bad in (dict(turned=4), dict(turned=72), dict(positions=0), dict(positions=1 << 31), dict(d_table=None), dict(d_table=A + 8)):
        assert append(call, r=rotation(**bad)) == ibp.IBP_EINVAL
    for odd in ("lens", "nxt", "w", "p"):
        assert append(call, **{odd: A + 1}) == ibp.IBP_EINVAL
    many = dict(k=rows(1 << 23), v=rows(1 << 23), q=None, q_out=None)
    assert append(call, **many) == ibp.IBP_EINVAL                                       # more blocks than a launch has
    none = dict(k=rows(0), v=rows(0), q=None, q_out=None)
    assert append(call, **none) == ibp.IBP_OK and append(call, n=0, **none) == ibp.IBP_OK
    assert append(call, n=0, lens=None, nxt=None, q=None, q_out=None) == ibp.IBP_OK     # rows outside all sequences


def test_read_refuses():
    for null in ("a", "g", "lens", "k", "v"):
        assert read(**{null: None}) == ibp.IBP_EINVAL
    assert read(v=rows(7)) == ibp.IBP_EINVAL and read(starts=None) == ibp.IBP_EINVAL and read(first=A + 2) == ibp.IBP_EINVAL
    assert read(k=rows(1 << 23), v=rows(1 << 23)) == ibp.IBP_EINVAL
    assert read(k=rows(0), v=rows(0)) == ibp.IBP_OK and read(n=0) == ibp.IBP_OK


def test_decode_refuses():
    assert decode(a=attn(flags=1)) == ibp.IBP_EINVAL
    assert decode(g=None) == ibp.IBP_EINVAL and decode(lens=None) == ibp.IBP_EINVAL
    assert decode(max_len=33) == ibp.IBP_ERANGE and decode(out=rows(7, heads=4)) == ibp.IBP_ENOMEM
    assert decode(w=A, ws=19) == ibp.IBP_ENOMEM
    need = ctypes.c_uint64(0)
    assert status("ibp_attn_decode4_workspace", 8, 4, 2, 64, 20, 1, need) == ibp.IBP_OK and need.value > 0
    assert decode(w=A, ws=20, s=None) == ibp.IBP_EINVAL and decode(w=A, ws=20, s=A + 8) == ibp.IBP_EINVAL
    assert decode(w=A, ws=20, sb=16) == ibp.IBP_ENOMEM
    assert decode(q=rows(0, heads=4), out=rows(0, heads=4), w=A, ws=20) == ibp.IBP_OK
    for bad in ((8, 4, 3, 64, 20, 0), (8, 4, 2, 60, 20, 0), (8, 4, 2, 64, 0x7fffffff, 0), (8, 4, 2, 264, 20, 0)):
        assert status("ibp_attn_decode4_workspace", *bad, need) == ibp.IBP_EINVAL
    assert status("ibp_attn_decode4_workspace", 8, 4, 2, 64, 20, 1, None) == ibp.IBP_EINVAL


@pytest.mark.parametrize("bad", [dict(row_stride=0), dict(head_stride=0), dict(row_stride=56), dict(head_stride=56)], ids=name)
def test_outputs_that_lie_in_themselves_are_refused(bad):
    """An expanded tensor has a stride of 0: as an input it is read, as an output two rows would be one."""
    four = rows(heads=4, **bad)
    for call in ("ibp_kv_append", "ibp_kv4_append"):
        assert append(call, q=four, q_out=four) == ibp.IBP_EINVAL and append(call, q_out=rows(heads=4, data=2 * A, **bad)) == ibp.IBP_EINVAL
        none = dict(k=rows(0), v=rows(0), q=rows(0, heads=4, row_stride=0), q_out=rows(0, heads=4, row_stride=0))
        assert append(call, **none) == ibp.IBP_OK
    assert read(k=rows(**bad)) == ibp.IBP_EINVAL and read(v=rows(**bad)) == ibp.IBP_EINVAL
    assert decode(q=four, out=four) == ibp.IBP_EINVAL
    one = dict(k=rows(0), v=rows(0), q=None, q_out=None)
    wide = lambda x: {k: bad["row_stride"] if "row_stride" in bad else bad["head_stride"] for k in x}  # noqa: E731
    for which in ("kp", "kh", "kt", "vp", "vh", "vt"):
        assert append(g=pages(**wide([which])), **one) == ibp.IBP_EINVAL
        assert append("ibp_kv4_append", g=pages(**{**wide([which]), which: min(wide([which])[which], 16)}), **one) == ibp.IBP_EINVAL
    assert append(g=pages(n_pages=1, page_tokens=1, kp=0, kt=0, vp=0, vt=0), **one) == ibp.IBP_OK


OVERLAPS = [dict(row_stride=64, head_stride=64), dict(row_stride=128, head_stride=64), dict(row_stride=192, head_stride=128),
            dict(row_stride=64, head_stride=448), dict(row_stride=72, head_stride=64)]


@pytest.mark.parametrize("bad", OVERLAPS, ids=name)
def test_rows_and_heads_that_lie_in_each_other_are_refused(bad):
    """Strides that hold a head each, by which one row's head is another row's: eight rows of four heads of 64."""
    four = rows(heads=4, **bad)
    heads4 = attn(kv_heads=4)
    for call in ("ibp_kv_append", "ibp_kv4_append"):
        none = dict(n=0, lens=None, nxt=None, starts=A)                   # (nothing would be launched)
        assert append(call, q=four, q_out=four, **none) == ibp.IBP_EINVAL
        assert append(call, q_out=rows(heads=4, data=2 * A, **bad), **none) == ibp.IBP_EINVAL
        assert append(call, a=heads4, q=None, q_out=None, k=four, v=four, g=pages(n_pages=0), **none) == ibp.IBP_OK      # read alone
    assert read(a=heads4, n=0, k=four, v=rows(heads=4)) == ibp.IBP_EINVAL and read(a=heads4, n=0, v=four, k=rows(heads=4)) == ibp.IBP_EINVAL
    assert decode(q=four, out=four) == ibp.IBP_EINVAL


BAD_POOLS = [dict(kp=64), dict(kp=1024), dict(kp=1984), dict(kh=512), dict(kt=128), dict(vp=1088), dict(vh=64, vt=64), dict(kp=1 << 40, kh=1 << 39, kt=1 << 39)]


@pytest.mark.parametrize("bad", BAD_POOLS, ids=name)
def test_pools_that_lie_in_themselves_are_refused(bad):
    none = dict(n=0, lens=None, nxt=None, q=None, q_out=None)
    assert append(g=pages(**bad), **none) == ibp.IBP_EINVAL
    four = {k: x // 64 * 24 if x < 1 << 39 else x for k, x in {**dict(kp=2048, kh=1024, kt=64, vp=2048, vh=1024, vt=64), **bad}.items()}
    assert append("ibp_kv4_append", g=pages(**four), **none) == ibp.IBP_EINVAL


def test_layouts_that_lie_apart_are_taken():
    """Any order of rows and heads, or of pages, heads and slots; keys and values in turns; padding; single ones of any stride."""
    none = dict(n=0, lens=None, nxt=None)
    for good in (dict(row_stride=256, head_stride=64), dict(row_stride=64, head_stride=512), dict(row_stride=320, head_stride=72),
                 dict(row_stride=1 << 23, head_stride=64), dict(row_stride=64, head_stride=1 << 40)):
        four = rows(heads=4, **good)
        for call in ("ibp_kv_append", "ibp_kv4_append"):
            assert append(call, q=four, q_out=four, g=pages(n_pages=0), **none) == ibp.IBP_OK
        assert read(a=attn(kv_heads=4), n=0, k=four, v=four) == ibp.IBP_OK
    assert append(q=rows(1, heads=4, row_stride=0), q_out=rows(1, heads=4, row_stride=0), k=rows(1), v=rows(1), **none) == ibp.IBP_OK
    assert append(a=attn(q_heads=1, kv_heads=1), q=rows(heads=1, head_stride=0), q_out=rows(heads=1, head_stride=0), **none) == ibp.IBP_OK
    orders = [dict(p=2048, h=1024, t=64), dict(p=2048, h=64, t=128), dict(p=4096, h=64, t=256), dict(p=64, h=256, t=512), dict(p=64, t=256, h=4096),
              dict(p=1024, h=4096, t=64), dict(p=4096, h=1152, t=72), dict(p=1 << 40, h=1 << 39, t=64)]
    for o in orders:
        assert append(g=pages(**{"k" + d: x for d, x in o.items()}, **{"v" + d: x for d, x in o.items()}), q=None, q_out=None, **none) == ibp.IBP_OK
    # (the largest counts and strides do not wrap around)
    assert append(g=pages(n_pages=0x7fffff00, page_tokens=1 << 24, kp=1 << 40, kh=1 << 39, vp=1 << 40, vh=1 << 39), q=None, q_out=None, **none) == ibp.IBP_OK
    assert append(g=pages(n_pages=0x7fffff00, page_tokens=1 << 24, kp=1 << 39, kh=1 << 40), q=None, q_out=None, **none) == ibp.IBP_EINVAL


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim", [(32, 8, 128), (8, 1, 256), (6, 2, 64), (16, 16, 80), (600, 600, 8), (64, 1, 128)])
def test_decode_workspace_is_enough_for_smaller_calls(heads, kv_heads, dim, weights):
    lens = sorted({128 * n + d for n in range(1, 140) for d in (-1, 0, 1)} | {1 << n for n in range(31)} | {3 << n for n in range(29)} | {0})
    need = lambda n, m: ibp.ibp_attn_decode4_workspace(n, heads, kv_heads, dim, m, weights)  # noqa: E731
    growing = lambda x: all(a <= b for a, b in zip(x, x[1:]))  # noqa: E731
    for n in (1, 2, 3, 5, 24, 64):
        assert growing([need(n, m) for m in lens])
    for m in (100, 513, 5500, 8193, 131071):
        assert growing([need(n, m) for n in range(80)])


def test_record_sizes():
    for dim in range(8, 257, 8):
        assert ibp.ibp_kv4_record(dim) == record_bytes(dim) >= 20 * -(-dim // 32) and record_bytes(dim) % 16 == 0
    assert [ibp.ibp_kv4_record(d) for d in (8, 32, 64, 128, 256)] == [32, 32, 48, 80, 160]
    out = ctypes.c_uint32(0)
    for bad in (0, 4, 12, 264):
        assert status("ibp_kv4_record", bad, out) == ibp.IBP_EINVAL
    assert status("ibp_kv4_record", 8, None) == ibp.IBP_EINVAL
    for bad in (-1, (1 << 32) + 64):
        with pytest.raises(ValueError):
            ibp.ibp_kv4_record(bad)


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [8, 40, 64, 128])
def test_records_hold_values_to_half_a_step(kind, dim):
    """Of the reference that the kernels are held to, bit for bit."""
    g = torch.Generator().manual_seed(dim)
    for spread in (1e-3, 1.0, 300.0):
        x = (torch.randn(200, dim, generator=g) * spread).to(kind)
        x[:20] += 5 * spread
        x[20:30] = x[20:30, :1]
        x[30:40, dim // 2] = 40 * spread
        r = records_of(x.float(), kind)
        off = (values_of(r, dim, kind) - x.double()).abs()
        # (a float16 step or centre below 2^-14 is off by up to 2^-25)
        assert (off <= held_bound(x, r, kind) + (2.0 ** -21 if kind == torch.float16 else 0)).all()


def test_binding_refuses_host_tensors():
    k, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    pool, pool4 = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(4, 2, 16, 48, dtype=torch.uint8)
    for call, p in (("ibp_kv_append", pool), ("ibp_kv4_append", pool4)):
        with pytest.raises(TypeError):
            getattr(ibp, call)(k, k, p, p, i[:, None], i, i)
    with pytest.raises(TypeError):
        ibp.ibp_kv4_read(pool4, pool4, i[:, None], i, k, k)
    with pytest.raises(TypeError):
        ibp.ibp_attn_decode4(k, pool4, pool4, i[:, None], i, 16, k)


@pytest.mark.parametrize("first", ["from paper_2605_30728_amd.kv_cache import ibp_kv4_record as f", "import paper_2605_30728_amd as ibp; f = ibp.ibp_kv4_record"])
def test_the_operators_are_reached_from_module_and_package(first):
    root = os.path.dirname(os.path.dirname(os.path.abspath(ibp.__file__)))
    done = subprocess.run([sys.executable, "-c", f"{first}; print(f(128))"], cwd=root, capture_output=True, text=True)
    assert (done.returncode, done.stdout.strip()) == (0, "80"), done.stderr


def test_the_module_needs_no_private_name_of_torch():
    """What a torch without GPU support may lack is asked for when it is there, and the public calls otherwise."""
    code = """
import torch
for name in [x for x in ("_cuda_getCurrentRawStream", "_cuda_getDevice") if hasattr(torch._C, x)]:
    delattr(torch._C, name)
import paper_2605_30728_amd as ibp
from paper_2605_30728_amd import kv_cache as kc
print(ibp.ibp_kv4_record(128), kc.ibp_kv_append is ibp.ibp_kv_append)
k = torch.zeros(1, 1, 8, dtype=torch.bfloat16)
i = torch.zeros(1, 1, dtype=torch.int32)
try:
    ibp.ibp_kv_append(k, k, k[None], k[None], i, i[0], i[0])
except TypeError as e:
    print(e)
class Stream:
    cuda_stream = 77
torch.cuda.current_stream = lambda device: Stream
print(kc._raw_stream(0))
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(ibp.__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert (done.returncode, done.stdout.splitlines()) == (0, ["80 True", "k must be a GPU tensor", "77"]), done.stderr


def test_binding_refuses_counts_beyond_32_bits():
    """Shapes alone (meta tensors have no data): a count that the library takes in 32 bits is neither cut nor an error of the packing."""
    def meta(*shape, kind=torch.int32):
        return torch.empty(shape, dtype=kind, device="meta")
    big = (1 << 32) + 1
    with pytest.raises(ValueError, match="sequences must fit 32 bits"):
        kc._sequences(big, meta(big), meta(big + 1), 5, -1)
    with pytest.raises(ValueError, match="sequences must fit 32 bits"):
        kc._sequences(big, meta(big), None, big, -1)
    kc._sequences(7, meta(7), meta(8), 5, -1)

    def pool(page, pages):
        x = meta(1, 1, page, 32, kind=torch.uint8)
        return kc._pool_of(x, x, meta(2, pages), -1, torch.uint8, 2, 1, 32, "records")
    assert pool((1 << 32) - 1, 1)[0] == pool(1, (1 << 32) - 1)[0] == 2
    for page, pages in ((1 << 32, 1), (1, 1 << 32)):
        with pytest.raises(ValueError, match="32 bits"):
            pool(page, pages)
