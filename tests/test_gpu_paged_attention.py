"""paged_attention against 64 bits: lengths, pages, head layouts, types, several tokens, rows that must not count, replays."""
import numpy as np
import pytest
import torch

from pages import TYPE, Pool, attention
from paper_2603_11243_amd.binding import Context, KvPages, SsdError

pytestmark = pytest.mark.gpu

# (queries, pages)
PAIRS = [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("f16", "e4m3"), ("bf16", "e4m3"), ("f32", "e4m3"), ("f16", "i8"), ("bf16", "i8"), ("f32", "i8")]
# (query heads, K/V heads, head_dim)
HEADS = [(16, 8, 128), (24, 8, 128), (4, 4, 64), (14, 2, 64), (5, 1, 128), (40, 2, 64)]
HEADS_32 = HEADS + [(3, 1, 4), (8, 2, 36), (2, 1, 100)]


def _context(B, n_new, heads, most):
    c = Context(device="cuda:0")
    c.reserve(paged_utts=B, paged_new=n_new, paged_ctx=most, paged_heads=heads)
    return c


def _queries(dtype, B, n_new, heads, seed=0, gap=0, scale=1.5):
    hq, _, hd = heads
    q = torch.full((B, n_new, hq * hd + gap), float("nan"), dtype=TYPE[dtype])
    q[..., :hq * hd] = (torch.randn(B, n_new, hq * hd, generator=torch.Generator().manual_seed(seed + 77)) * scale).to(TYPE[dtype])
    return q.cuda()[..., :hq * hd].unflatten(2, (hq, hd))


def _check(pair, heads, ctx_len, page_rows=16, n_new=1, seed=0, gap=0, scale=None, change=None, lost=lambda b, j: False, flags=0, most=None, ctx=None, pool=None, **more):
    q = _queries(pair[0], len(ctx_len), n_new, heads, seed, gap)
    pool = pool or Pool(pair[1], heads[1:], ctx_len, page_rows, seed, most=most)
    c = ctx or _context(len(ctx_len), n_new, heads, pool.table.shape[1] * page_rows)
    want, tol, want_lse, lse_tol = attention(q, pool, n_new, scale, lost)
    if change:
        change(q, pool)
    lse = torch.full(q.shape[:3], 7.0, device="cuda")
    c.device_flags()
    out = c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len, scale=scale, lse=lse, **more)
    torch.cuda.synchronize()
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    off = np.abs(got - want) - tol
    assert got.shape == want.shape and np.isfinite(got).all() and (off <= 0).all(), (np.argwhere(~(off <= 0))[:5], off.max(), tol.mean())
    nothing = np.isinf(want_lse)
    assert np.array_equal(nothing, np.isneginf(got_lse))
    assert (np.abs(got_lse[~nothing] - want_lse[~nothing]) <= lse_tol[~nothing]).all()
    assert c.device_flags() == flags
    if ctx is None:
        c.close()
    return out


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page_rows, n_new", [(16, 1), (64, 1), (32, 3), (256, 5)])
def test_ragged_batches(pair, heads, page_rows, n_new):
    _check(pair, heads, [0, 1, 2, 15, 16, 17, 31, 33, 64, 65, 130, 200], page_rows, n_new)


@pytest.mark.parametrize("heads", HEADS_32[len(HEADS):])
@pytest.mark.parametrize("n_new", [1, 7])
def test_head_dims_of_fp32(heads, n_new):
    _check(("f32", "f32"), heads, [0, 1, 16, 40, 300, 77], 32, n_new)


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("n", [1, 127, 128, 129, 255, 256, 257, 511, 513, 1000, 2047, 2049, 4096, 4097, 9001])
def test_lengths(pair, n):
    _check(pair, (4, 2, 128), [n, max(1, n // 3)], 64)


@pytest.mark.parametrize("pair", [("f16", "f16"), ("bf16", "e4m3"), ("f16", "i8"), ("f32", "f32")])
@pytest.mark.parametrize("n_new", [2, 8, 9, 17, 40])
@pytest.mark.parametrize("heads", [(4, 2, 64), (24, 8, 128), (3, 3, 128)])
def test_several_tokens(pair, n_new, heads):
    """More query rows than one tile holds; tokens that see nothing, in contexts shorter than the new tokens."""
    _check(pair, heads, [0, 1, n_new - 1, n_new, n_new + 1, 64, 600], 16, n_new)


@pytest.mark.parametrize("pair", [("f16", "f16"), ("bf16", "i8"), ("f32", "f32"), ("f32", "e4m3")])
def test_many_query_heads(pair):
    _check(pair, (512, 1, 64), [70, 3], 16)
    _check(pair, (100, 4, 64), [40], 32, 3)


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0, 1e-20])
def test_scales(pair, scale):
    _check(pair, (4, 2, 64), [50, 300], 16, 2, scale=scale)


@pytest.mark.parametrize("pair", PAIRS)
def test_strided_queries(pair):
    _check(pair, (4, 2, 64), [50, 30, 9], 16, 2, gap=192)
    q = _queries(pair[0], 3, 1, (4, 2, 64), gap=64)[:, 0]
    pool, c = Pool(pair[1], (2, 64), [50, 30, 9], 16), _context(3, 1, (4, 2, 64), 64)
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    assert c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len, out=out) is out
    want, tol, _, _ = attention(q[:, None], pool, 1)
    assert (np.abs(out.double().cpu().numpy() - want[:, 0]) <= tol[:, 0]).all()


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_rows_of_later_tokens_do_not_count(pair, bad):
    """The last row is not finite: only the last token is touched."""
    heads, n_new = (4, 2, 64), 4
    q, pool = _queries(pair[0], 2, n_new, heads), Pool(pair[1], heads[1:], [50, 67], 16)
    want, tol, _, _ = attention(q, pool, n_new)
    for b in range(2):
        j = int(pool.ctx_host[b]) - 1
        at = (0, int(pool.table_host[b, j // 16]), slice(None), j % 16)
        for name in ("k", "v"):
            if pool.kind in ("e4m3", "i8"):
                pool.parts[name + "_scale"][at] = float(bad)
                if pool.kind == "e4m3" and bad == "nan":
                    pool.parts[name].view(torch.uint8)[at] = 127
            else:
                pool.parts[name][at] = float(bad)
    c = _context(2, n_new, heads, 80)
    out = c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len).double().cpu().numpy()
    assert (np.abs(out - want) <= tol)[:, :-1].all()
    assert not np.isfinite(out[:, -1]).any()


@pytest.mark.parametrize("pair", [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32")])
def test_a_seen_value_that_is_not_finite_stays_in_its_column(pair):
    for n in (40, 3000):
        heads = (4, 2, 64)
        q, pool = _queries(pair[0], 1, 2, heads), Pool(pair[1], heads[1:], [n], 16)
        want, tol, _, _ = attention(q, pool, 2)
        for j, d, x in ((n - 5, 7, "nan"), (3, 20, "inf"), (n - 20, 33, "-inf")):
            pool.parts["v"][0, int(pool.table_host[0, j // 16]), 1, j % 16, d] = float(x)
        out = _context(1, 2, heads, n + 16).paged_attention(q, pool.pages(), pool.table, pool.ctx_len).double().cpu().numpy()
        touched = np.zeros(want.shape, dtype=bool)
        touched[:, :, 2:, [7, 20, 33]] = True
        assert not np.isfinite(out[touched]).any() and (np.abs(out - want) <= tol)[~touched].all()


@pytest.mark.parametrize("pair", PAIRS)
def test_pages_that_are_none(pair):
    """Their rows are not seen, also if none is left."""
    def change(q, pool):
        pool.table[0, 2] = -1
        pool.table[1, 0] = pool.n_pages
        pool.table[2, :] = -2 ** 31
    _check(pair, (4, 2, 64), [100, 20, 33, 50, 700], 16, 2, change=change, lost=lambda b, j: (b == 0 and 32 <= j < 48) or (b == 1 and j < 16) or b == 2, flags=4)


@pytest.mark.parametrize("pair", [("f16", "f16"), ("bf16", "e4m3"), ("f32", "f32")])
def test_lengths_out_of_range(pair):
    heads = (4, 2, 64)
    q, c = _queries(pair[0], 3, 1, heads), _context(3, 1, heads, 64)
    pool = Pool(pair[1], heads[1:], [64, 64, 0], 16)
    want, tol, _, _ = attention(q, pool, 1)
    pool.ctx_len.copy_(torch.tensor([65, 2 ** 31 - 1, -3]))
    c.device_flags()
    out = c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len).double().cpu().numpy()
    assert (np.abs(out - want) <= tol).all() and c.device_flags() == 4
    out = c.paged_attention(q, pool.pages(), pool.table[:, :0], torch.zeros_like(pool.ctx_len))
    assert (out == 0).all() and c.device_flags() == 0


def test_shared_pages():
    """Two utterances whose first rows are the same pages, and one list three times."""
    heads = (4, 2, 64)
    pool = Pool("e4m3", heads[1:], [100, 100, 37, 100, 100], 32)
    for b in (1, 3, 4):
        for j in range(2):
            pool.table_host[b, j] = pool.table_host[0, j]
    pool.table_host[4] = pool.table_host[0]
    pool.table.copy_(torch.from_numpy(pool.table_host))
    _check(("f16", "e4m3"), heads, [100, 100, 37, 100, 100], 32, pool=pool)


def test_no_precision_is_lost_between_equal_scores():
    """Means of many values of one magnitude in fp32 pages and by three-value weights: errors of fp32, not of 16 bits."""
    for pair in (("f32", "f32"), ("f32", "i8"), ("f32", "e4m3")):
        heads, n = (2, 2, 64), 5000
        pool = Pool(pair[1], heads[1:], [n], 64)
        q = _queries("f32", 1, 1, heads, scale=0.1)
        want, _, _, _ = attention(q, pool, 1)
        out = _context(1, 1, heads, n + 64).paged_attention(q, pool.pages(), pool.table, pool.ctx_len).double().cpu().numpy()
        assert np.linalg.norm(out - want) <= 2e-5 * np.linalg.norm(want)


@pytest.mark.parametrize("pair", [("bf16", "bf16"), ("f32", "f32"), ("f32", "i8"), ("bf16", "e4m3")])
def test_values_at_the_end_of_the_range(pair):
    """Sums of values whose mean is in fp32's range, though they themselves are not."""
    heads, n = (2, 2, 64), 700
    pool, q = Pool(pair[1], heads[1:], [n], 16), _queries(pair[0], 1, 1, heads, scale=0.1)
    if pair[1] in ("e4m3", "i8"):
        s = pool.parts["v_scale"]
        s.copy_(torch.where(s.isnan(), s, 2.0 ** 119 if pair[1] == "e4m3" else 2.0 ** 120))
        pool.parts["v"].view(torch.uint8).fill_(0x7c if pair[1] == "e4m3" else 100)
    else:
        v = pool.parts["v"]
        v.copy_(torch.where(v.isnan(), v, 3.2e38))
    want, tol, _, _ = attention(q, pool, 1)
    out = _context(1, 1, heads, n + 16).paged_attention(q, pool.pages(), pool.table, pool.ctx_len).double().cpu().numpy()
    assert (np.abs(out / 2.0 ** 64 - want / 2.0 ** 64) <= tol / 2.0 ** 64).all()


def test_pools_beyond_4_gib():
    H, hd, R, n = 8, 128, 64, 1000
    n_pages = (9 << 30) // (H * R * hd * 2)
    big = torch.zeros(n_pages, H, R, hd, dtype=torch.bfloat16, device="cuda")
    r = np.random.default_rng(0)
    order = r.permutation(n_pages - 20)[:14].tolist() + [n_pages - 1, n_pages - 2]
    table = torch.tensor([order], dtype=torch.int32, device="cuda")
    small = Pool("bf16", (H, hd), [n], R, seed=3)
    for j, page in enumerate(order):
        big[page] = small.parts["k"][0, int(small.table_host[0, j])].nan_to_num()
    q = _queries("bf16", 1, 1, (16, H, hd))
    small.parts["v"] = small.parts["k"]
    want, tol, _, _ = attention(q, small, 1)
    out = _context(1, 1, (16, H, hd), 1024).paged_attention(q, KvPages(big, big), table, small.ctx_len).double().cpu().numpy()
    assert (np.abs(out - want) <= tol).all()


def test_repeats_to_the_bit_and_batches_do_not_mix():
    """Twice the same; an utterance by itself, in the same launch shape, too."""
    heads = (16, 8, 128)
    pool = Pool("i8", heads[1:], [3000, 40, 777, 0, 2048], 64)
    q, c = _queries("f16", 5, 2, heads), _context(5, 2, heads, 3200)
    a = c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len)
    for _ in range(3):
        assert torch.equal(a, c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len))
    swapped = c.paged_attention(q.flip(0).contiguous(), pool.pages(), pool.table.flip(0).contiguous(), pool.ctx_len.flip(0).contiguous())
    assert torch.equal(a, swapped.flip(0))


@pytest.mark.parametrize("pair", [("f16", "f16"), ("bf16", "e4m3"), ("f32", "f32")])
@pytest.mark.parametrize("lens, most", [([3000, 5], 100000), ([700] * 9, 30000), ([0] * 63 + [2500], 2600), ([1], 1 << 20)])
def test_tables_far_longer_than_the_contexts(pair, lens, most):
    """What a captured step is made for: the pieces go by the lengths, not by what the table could hold."""
    _check(pair, (4, 2, 64), lens, 64, 2, most=most)


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("hd", [64, 128])
def test_wide_tiles(pair, hd):
    """What long contexts take where there are more than 16 query rows, over short ones too: the launch is made for 400000 rows."""
    _check(pair, (8, 2, hd), [0, 5, 300, 2000, 8], 64, 9, most=400000)


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_rows_of_later_tokens_do_not_count_in_wide_tiles(pair, bad):
    """The last row but two is not finite: tokens before it stay as they are, columns of either half of a tile."""
    heads, n_new = (8, 2, 128), 9
    q, pool = _queries(pair[0], 2, n_new, heads), Pool(pair[1], heads[1:], [50, 667], 16, most=400000)
    want, tol, _, _ = attention(q, pool, n_new)
    for b in range(2):
        j = int(pool.ctx_host[b]) - 3
        at = (0, int(pool.table_host[b, j // 16]), slice(None), j % 16)
        for name in ("k", "v"):
            if pool.kind in ("e4m3", "i8"):
                pool.parts[name + "_scale"][at] = float(bad)
                if pool.kind == "e4m3" and bad == "nan":
                    pool.parts[name].view(torch.uint8)[at] = 127
            else:
                pool.parts[name][at] = float(bad)
    out = _context(2, n_new, heads, 400000).paged_attention(q, pool.pages(), pool.table, pool.ctx_len).double().cpu().numpy()
    assert (np.abs(out - want) <= tol)[:, :-3].all()
    assert not np.isfinite(out[:, -3:]).any()


@pytest.mark.parametrize("B, long", [(65, 900), (70, 3000), (300, 2500), (1024, 4200), (1030, 4200), (1030, 9000)])
def test_large_batches_with_one_long_context(B, long):
    lens = [b % 7 for b in range(B)]
    lens[B // 2] = long
    lens[B - 1] = long - 300
    _check(("f16", "e4m3"), (2, 1, 64), lens, 16)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("B", [2, 7, 33])
def test_ragged_long_contexts(hd, B):
    """Every piece in its place: contexts from nothing to many pieces."""
    r = np.random.default_rng(B)
    lens = [int(n) for n in np.exp(r.uniform(0, np.log(6000), B))]
    lens[0], lens[-1] = 0, 6000
    _check(("bf16", "i8"), (6, 2, hd), lens, 128, 3)


@pytest.mark.parametrize("kind", ["f16", "e4m3", "i8"])
def test_a_captured_decoding_loop(kind):
    """Append and attend, captured once and replayed while contexts grow over pages and are replaced: the eager results, with eager work of the program between replays."""
    heads, B, R = (4, 2, 64), 3, 16
    side = torch.cuda.Stream()
    c, eager = Context(device="cuda:0", stream=side), Context(device="cuda:0", stream=side)
    for x in (c, eager):
        x.reserve(paged_utts=B, paged_new=1, paged_ctx=1600, paged_heads=heads)
    pool = Pool(kind, heads[1:], [14, 700, 1590], R, most=1600)
    with torch.cuda.stream(side):
        free = [p for p in range(pool.n_pages) if p not in set(pool.table_host[pool.table_host >= 0].tolist())]
        table, n = pool.table.clone().clamp_(min=-1), pool.ctx_len.clone()
        table[0, 1], table[1, 44] = free                     # the pages that contexts of 14 and 700 rows grow into
        q, k, v = (torch.randn(B, h, 64, device="cuda").half() for h in (4, 2, 2))
        out, want = torch.empty_like(q), torch.empty_like(q)
        pages, other = pool.pages(), KvPages(*(None if t is None else t.clone() for t in (pool.parts["k"], pool.parts["v"], pool.parts.get("k_scale"), pool.parts.get("v_scale"))))
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            c.kv_write_pages(pages, table, n, k, v, max_ctx=1600)
            c.paged_attention(q, pages.layer(0), table, n, max_ctx=1600, out=out)
        for step in range(12):
            for t in (q, k, v):
                t.copy_(torch.randn(t.shape))
            graph.replay()
            eager.kv_write_pages(other, table, n, k, v, max_ctx=1600)
            eager.paged_attention(q, other.layer(0), table, n, max_ctx=1600, out=want)
            side.synchronize()
            assert torch.equal(out, want) and torch.isfinite(out).all(), step
            assert torch.equal(pages.k.view(torch.uint8), other.k.view(torch.uint8))
            n.add_(torch.tensor([1, 1, 0 if step > 8 else 1], dtype=torch.int32, device="cuda"))
    assert c.device_flags() == 0
    for x in (c, eager):
        x.close()


def test_other_streams():
    """The context's stream does the work, whichever is current; results are in order there."""
    heads = (4, 2, 64)
    side = torch.cuda.Stream()
    c = Context(device="cuda:0", stream=side)
    c.reserve(paged_utts=2, paged_new=1, paged_ctx=2048, paged_heads=heads)
    pool, q = Pool("e4m3", heads[1:], [2000, 900], 64), _queries("bf16", 2, 1, heads)
    want, tol, _, _ = attention(q[:, :], pool, 1)
    torch.cuda.synchronize()
    out = c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len)
    side.synchronize()
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    c.close()


def test_refusals_of_the_binding():
    heads = (4, 2, 64)
    c, pool, q = _context(2, 1, heads, 64), Pool("i8", heads[1:], [60, 20], 16), _queries("f16", 2, 1, heads)
    call = lambda q=q, pages=pool.pages(), table=pool.table, n=pool.ctx_len, **k: c.paged_attention(q, pages, table, n, **k)
    call()
    for bad in (dict(q=q[:1]), dict(q=q.double()), dict(q=torch.empty(2, 1, 64, 4, dtype=q.dtype, device="cuda").transpose(2, 3)), dict(q=q[..., :32]), dict(table=pool.table.long()), dict(table=pool.table.cpu()), dict(table=pool.table[0]),
                dict(n=pool.ctx_len[:1]), dict(n=pool.ctx_len.long()), dict(n=pool.ctx_len.cpu()), dict(max_ctx=65), dict(out=torch.empty(3, device="cuda")),
                dict(out=torch.empty(q.numel() + 64, dtype=q.dtype, device="cuda")), dict(lse=torch.empty(3, device="cuda")), dict(q=q.cpu())):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(q=q[:, :0]), dict(max_ctx=-1), dict(scale=float("inf")), dict(out=q)):
        with pytest.raises(SsdError):
            call(**bad)
    with pytest.raises(SsdError):
        call(q=q[..., :3, :])
    moves = lambda **k: c.kv_write_pages(**{**dict(pages=pool.pages(), page_table=pool.table, ctx_len=pool.ctx_len, k=torch.zeros(1, 8, 2, 64, device="cuda"),
                                                   v=torch.zeros(1, 8, 2, 64, device="cuda"), max_rows=4), **k})
    moves()
    moves(max_rows=None)
    for bad in (dict(start=pool.ctx_len.long()), dict(start=pool.ctx_len[:1]), dict(n_rows=pool.ctx_len.cpu()), dict(max_rows=None, start=pool.ctx_len),
                dict(k=torch.zeros(1, 7, 2, 64, device="cuda"), v=torch.zeros(1, 7, 2, 64, device="cuda"), max_rows=None), dict(max_ctx=65)):
        with pytest.raises(ValueError):
            moves(**bad)
    with pytest.raises(SsdError):
        moves(max_rows=5)


@pytest.mark.parametrize("pair", [("f16", "f16"), ("bf16", "i8"), ("f32", "e4m3"), ("f32", "f32")])
@pytest.mark.parametrize("heads, lens", [((8, 1, 128), [30000]), ((16, 4, 64), [9000, 8000, 127]), ((8, 4, 128), [5000] * 7 + [1]), ((6, 6, 64), [4000] * 20)])
def test_joining_few_and_many_pieces(pair, heads, lens):
    """About 235, 70, 20 and 8 pieces a context, and one with a piece or two beside them; the first token sees one row less."""
    _check(pair, heads, lens, 128, 2)


@pytest.mark.parametrize("pair", [("f32", "e4m3"), ("f32", "i8"), ("bf16", "i8"), ("bf16", "e4m3"), ("f32", "f32"), ("bf16", "bf16")])
def test_large_queries(pair):
    """Queries times a power of two and the scale divided by it: every product and sum is the same but for its exponent, and so every output is the same to the bit."""
    heads = (8, 2, 128)
    pool = Pool(pair[1], heads[1:], [700, 3, 64], 32)
    q, c = _queries(pair[0], 3, 3, heads), _context(3, 3, heads, pool.table.shape[1] * 32)
    want = c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len, scale=0.0625)
    got = c.paged_attention(q * 2.0 ** 100, pool.pages(), pool.table, pool.ctx_len, scale=0.0625 * 2.0 ** -100)
    assert torch.equal(got, want) and c.device_flags() == 0
    c.close()
