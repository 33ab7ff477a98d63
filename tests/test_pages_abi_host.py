"""kv_write_pages, kv_read_pages and paged_attention refuse bad arguments on the host (no GPU: no pointer is followed)."""
import ctypes as C
import os

import pytest

from test_tree_abi_host import BF16, EINVAL, ESHAPE, EUNSUPPORTED, EWORKSPACE, F16, F32, ctx, lib, view  # noqa: F401

E4M3, I8 = 3, 4
K, V, KS, VS = 1 << 44, 1 << 45, 1 << 46, 1 << 47
TABLE, LEN, Q, OUT, LSE = 1 << 20, 1 << 21, 1 << 24, 1 << 26, 1 << 27


class PagesC(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("pages", C.c_int64), ("page_rows", C.c_int32),
                ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32)]


class TableC(C.Structure):
    _fields_ = [("entries", C.c_void_p), ("stride", C.c_int64), ("ctx_len", C.c_void_p), ("B", C.c_int32), ("max_ctx", C.c_int32)]


def pages(k=K, v=V, ks=None, vs=None, n=1000, R=16, L=1, H=2, hd=128, dtype=F16):
    eight = dtype in (E4M3, I8)
    return PagesC(k, v, (KS if eight else 0) if ks is None else ks, (VS if eight else 0) if vs is None else vs, n, R, L, H, hd, dtype)


def table(entries=TABLE, stride=10, ctx_len=LEN, B=3, max_ctx=160):
    return TableC(entries, stride, ctx_len, B, max_ctx)


def ref(x):
    return None if x is None else C.byref(x)


def attention(lib, ctx, q=Q, dtype=F16, q_stride=512, hq=4, n_new=1, p=(), t=(), scale=0.1, out=OUT, lse=None):
    return lib.paged_attention(ctx, q, dtype, q_stride, hq, n_new, ref(pages() if p == () else p), ref(table() if t == () else t), C.c_float(scale), out, lse)


def both(lib, ctx, slots=(), start=None, n_rows=None, most=20, p=(), t=()):
    s, p, t = ref(view() if slots == () else slots), ref(pages(dtype=I8) if p == () else p), ref(table() if t == () else t)
    rc = {lib.kv_write_pages(ctx, s, start, n_rows, most, p, t), lib.kv_read_pages(ctx, p, t, s, start, n_rows, most)}
    assert len(rc) == 1, rc
    return rc.pop()


BAD_PAGES = [(EINVAL, k) for k in ({"k": 0}, {"v": 0}, {"k": K + 8}, {"v": V + 4}, {"ks": 0}, {"vs": 0}, {"ks": KS + 4}, {"n": 0}, {"n": 1 << 31}, {"L": 0}, {"H": 0}, {"hd": 0})] + \
    [(ESHAPE, k) for k in ({"R": 0}, {"R": 8}, {"R": 48}, {"R": 512}, {"hd": 32}, {"hd": 96}, {"hd": 256}, {"H": 65536}, {"L": 40000, "H": 2}, {"n": (1 << 31) - 1, "H": 4096, "R": 256})] + \
    [(EUNSUPPORTED, {"dtype": 5}), (EUNSUPPORTED, {"dtype": -1})]
BAD_TABLES = [(EINVAL, k) for k in ({"entries": 0}, {"ctx_len": 0}, {"B": 0}, {"B": -1}, {"max_ctx": -1}, {"max_ctx": (1 << 30) + 1}, {"stride": 9}, {"stride": -10}, {"max_ctx": 161})] + \
    [(ESHAPE, {"B": 65536})]


@pytest.mark.parametrize("want, more", BAD_PAGES)
def test_pages(lib, ctx, want, more):  # noqa: F811
    assert attention(lib, ctx, p=pages(**{"dtype": I8, **more})) == want, lib.ssd_last_error(ctx)
    fits = {k: x for k, x in more.items() if k in ("L", "H", "hd")}
    if not fits:
        assert both(lib, ctx, p=pages(**{"dtype": I8, **more})) == want, lib.ssd_last_error(ctx)


@pytest.mark.parametrize("want, more", BAD_TABLES)
def test_tables(lib, ctx, want, more):  # noqa: F811
    assert attention(lib, ctx, t=table(**more)) == want and both(lib, ctx, t=table(**more)) == want
    assert lib.ssd_last_error(ctx)


def test_null(lib, ctx):  # noqa: F811
    assert attention(lib, None) == EINVAL and both(lib, None) == EINVAL
    assert attention(lib, ctx, p=None) == EINVAL and attention(lib, ctx, t=None) == EINVAL
    assert both(lib, ctx, p=None) == EINVAL and both(lib, ctx, t=None) == EINVAL and both(lib, ctx, slots=None) == EINVAL


def test_attention(lib, ctx):  # noqa: F811
    call = lambda **k: attention(lib, ctx, **k)
    for k in ({"q": None}, {"out": None}, {"q": Q + 8}, {"out": OUT + 8}, {"q_stride": 511}, {"q_stride": 516}, {"n_new": 0}, {"n_new": -1}, {"p": pages(L=2)},
              {"scale": float("nan")}, {"scale": float("inf")}, {"scale": 3e38}):
        assert call(**k) == EINVAL, k
    for k in ({"hq": 3}, {"hq": 0}, {"hq": -2}, {"hq": 1026, "q_stride": 1 << 18}, {"n_new": 16 * 65536 // 2 // 3 + 16}):
        assert call(**k) == ESHAPE, k
    # 2^21 query heads of tokens: as many workgroups join the pieces
    many = dict(p=pages(H=64, dtype=I8), hq=64, q_stride=8192, q=1 << 50, out=1 << 52, t=table(B=512, stride=1000, max_ctx=16000))
    assert call(n_new=64, **many) == EWORKSPACE and call(n_new=65, **many) == ESHAPE
    for k in ({"dtype": 3}, {"dtype": 9}, {"dtype": BF16}, {"dtype": F32, "q_stride": 1024}, {"p": pages(dtype=F32)}, {"p": pages(dtype=BF16)}):
        assert call(**k) == EUNSUPPORTED, k
    for near in (0, 3 * 1024 - 16, -3 * 1024 + 16):
        assert call(out=Q + near) == EINVAL, near


def test_moves(lib, ctx):  # noqa: F811
    call = lambda **k: both(lib, ctx, **k)
    assert call(most=-1) == EINVAL
    assert call(most=34) == EINVAL and b"slots" in lib.ssd_last_error(ctx)              # 3 utterances of 34 rows in 100 slots
    for p in (pages(dtype=I8, H=1), pages(dtype=I8, hd=64), pages(dtype=I8, L=2)):
        assert call(p=p) == EINVAL
    for p, slots in ((pages(dtype=BF16), view()), (pages(dtype=F16), view(dtype=BF16)), (pages(dtype=F32), view()), (pages(dtype=F16), view(dtype=F32))):
        assert call(p=p, slots=slots) == EUNSUPPORTED
    assert call(slots=view(dtype=3)) == EUNSUPPORTED and call(slots=view(ss=260)) == EINVAL
    n = 1000 * 2 * 16 * 128                                                              # bytes of the pages, and of 1 << 40 the slots
    for p in (pages(dtype=I8, k=(1 << 40) - n + 16), pages(dtype=I8, v=(1 << 40) + 100 * 512 - 16), pages(dtype=I8, ks=(1 << 40) + 16),
              pages(dtype=I8, vs=(1 << 40) + (1 << 30))):
        assert call(p=p) == EINVAL and b"overlap" in lib.ssd_last_error(ctx)
    write = lambda p: lib.kv_write_pages(ctx, ref(view()), None, None, 20, ref(p), ref(table()))
    for p in (pages(dtype=I8, v=K), pages(dtype=I8, v=K + n - 16), pages(dtype=I8, ks=K + 16), pages(dtype=I8, vs=KS + 64)):
        assert write(p) == EINVAL
    assert lib.kv_read_pages(ctx, ref(pages(dtype=I8)), ref(table()), ref(view(v=1 << 40)), None, None, 20) == EINVAL
    for most in ((1 << 30) + 1, (1 << 31) - 1):
        assert lib.kv_write_pages(ctx, ref(view()), LEN, LEN, most, ref(pages(dtype=I8)), ref(table())) == EINVAL
        assert lib.kv_read_pages(ctx, ref(pages(dtype=I8)), ref(table()), ref(view()), LEN, LEN, most) == EINVAL
    # nothing to do is not an error
    assert call(most=0) == 0 and call(t=table(max_ctx=0, entries=0)) == 0


def test_workspace_sizes(lib, ctx):  # noqa: F811
    size = lambda *a: lib.ssd_paged_workspace_bytes(ctx, *a)
    assert size(0, 1, 1, 1, 1, 1) == 0 and size(16, 8, 128, -1, 1, 10) == 0 and lib.ssd_paged_workspace_bytes(None, 16, 8, 128, 1, 1, 10) == 0
    last = 0
    for n in (1, 100, 257, 3000, 70000, 1 << 20):
        for B in (1, 3, 64):
            for new in (1, 4, 9):
                assert size(16, 8, 128, B, new, n) >= size(16, 8, 128, 1, 1, n) >= last
        last = size(16, 8, 128, 1, 1, n)


def test_workspace_covers_every_call(lib, ctx):  # noqa: F811
    """What a call without a workspace says it needs is at most what ssd_paged_workspace_bytes says, and what that says for more of anything."""
    import random
    import re
    r = random.Random(1)
    some = lambda top: max(1, int(top ** r.random()))
    for _ in range(4000):
        B, new, H, G, n, hd = some(65535), some(300), some(64), some(64), some(1 << 30), r.choice([64, 128])
        if (new * G + 15) // 16 * B > 65535 or B * new * G * H > 1 << 21:
            continue
        rc = attention(lib, ctx, q=1 << 50, out=1 << 60, q_stride=G * H * hd, hq=G * H, n_new=new, p=pages(H=H, hd=hd, R=16), t=table(B=B, max_ctx=n, stride=1 << 27))
        need = 0
        if rc == EWORKSPACE:
            need = int(re.search(rb"workspace of (\d+) bytes", lib.ssd_last_error(ctx)).group(1))
            size = lambda *a: lib.ssd_paged_workspace_bytes(ctx, *a)
            assert need <= size(G * H, H, hd, B, new, n)
            for more in (size(G * H, H, hd, B + some(100), new, n), size(G * H, H, 128, B, new + some(10), min(1 << 30, n + some(10000))), size(2 * G * H, H, hd, B, new, n)):
                assert need <= more or more == 0                 # (0: no call is so large)
        else:
            assert n <= 4096 or rc != 0


def test_python_refusals():
    """What the binding sees before the library does."""
    import torch
    from paper_2603_11243_amd.binding import KvPages
    k = torch.zeros(4, 2, 16, 64, dtype=torch.float16)
    s = torch.zeros(4, 2, 16)
    KvPages(k, k.clone())
    codes = KvPages(k.to(torch.int8), k.to(torch.int8), s, s.clone())
    assert codes.n_pages == 4 and codes.n_kv_heads == 2 and codes.page_rows == 16 and codes.head_dim == 64 and codes.n_layers == 1 and codes.layer(0).k is codes.k
    for bad in ((k, k[:3]), (k, k.bfloat16()), (k, k.transpose(0, 1)), (k.double(), k.double()), (k, k, s, s), (k.to(torch.int8), k.to(torch.int8)),
                (k.to(torch.int8), k.to(torch.int8), s, None), (k.to(torch.int8), k.to(torch.int8), s, s.double()), (k.to(torch.int8), k.to(torch.int8), s[:3], s[:3]),
                (k[..., ::2], k[..., ::2]), (k[0], k[0])):
        with pytest.raises(ValueError):
            KvPages(*bad)
    with pytest.raises(IndexError):
        codes.layer(1)


def test_results_share_no_memory(lib, ctx):  # noqa: F811
    rows = 1000 * 2 * 16
    places = {"k": (K, rows * 128), "v": (V, rows * 128), "ks": (KS, rows * 4), "vs": (VS, rows * 4), "q": (Q, 3 * 512 * 2)}
    for name, (at, size) in places.items():
        for near in (at, at + size - 16, at - 16):
            for k in ({"out": near}, {"lse": near}):
                assert attention(lib, ctx, p=pages(dtype=I8), **k) == EINVAL and b"overlap" in lib.ssd_last_error(ctx), (name, k)
    for lse in (OUT, OUT + 3 * 512 * 2 - 16, OUT - 16):
        assert attention(lib, ctx, p=pages(dtype=I8), lse=lse) == EINVAL and b"overlap" in lib.ssd_last_error(ctx)


def test_no_call_without_flags(lib, ctx):  # noqa: F811
    """Without a GPU a context has none: nothing is launched, and the call says why."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("this context has flags")
    assert attention(lib, ctx) == -4 and b"flags" in lib.ssd_last_error(ctx)
    assert both(lib, ctx) == -4 and b"flags" in lib.ssd_last_error(ctx)
    flags = C.c_int32(7)
    assert lib.ssd_device_flags(ctx, C.byref(flags)) == 0 and flags.value == 0


@pytest.mark.parametrize("B, H, G, new", [(64, 8, 2, 1), (1, 8, 3, 9), (1024, 2, 1, 1), (20, 1, 64, 4)])
def test_shared_pieces_do_not_grow_with_the_table(lib, ctx, B, H, G, new):  # noqa: F811
    """What a call needs, and so what it launches, is by its utterances and heads: the same for tables of 2^16 rows an utterance and of 2^24."""
    import re
    need = []
    for bits in (16, 20, 24):
        rc = attention(lib, ctx, q=1 << 50, out=1 << 52, hq=H * G, q_stride=H * G * 128, n_new=new, p=pages(H=H, R=64), t=table(B=B, max_ctx=1 << bits, stride=1 << bits))
        assert rc == EWORKSPACE
        need.append(int(re.search(rb"workspace of (\d+) bytes", lib.ssd_last_error(ctx)).group(1)))
        assert need[-1] <= lib.ssd_paged_workspace_bytes(ctx, H * G, H, 128, B, new, 1 << bits) < (64 << 20) + 8 * 1024 * B * new * H * G
    assert need[0] == need[1] == need[2]
