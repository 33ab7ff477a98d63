"""kv_evict against its definition: which rows stay is exact, and they are copied as they are."""
import numpy as np
import pytest
import torch

from paper_2603_11243_amd.binding import Context

pytestmark = pytest.mark.gpu

DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _kept(mass, keep, first, recent):
    """Rows of one head by definition; NaN below everything, equal ones in order."""
    n = len(mass)
    if keep >= n:
        return list(range(n))
    key = np.where(np.isnan(mass), -np.inf, mass.astype(np.float64))
    order = sorted(range(first, n - recent), key=lambda i: (not np.isnan(mass[i]), key[i], -i), reverse=True)
    return sorted(list(range(first)) + order[:keep - first - recent] + list(range(n - recent, n)))


def _check(mass_of, dtype="f16", L=2, H=3, hd=64, ctx_len=(40,), keep=(17,), first=0, recent=0, layout="slots", want_rows=True, want_mass=True, seed=0,
           ctx=None):
    g, r = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
    B, ctx_len = len(ctx_len), np.array(ctx_len)
    kept = np.minimum(keep, ctx_len)

    def places(sizes):
        at, start = 2, np.zeros(B, dtype=np.int32)
        for b in r.permutation(B):
            start[b] = at
            at += int(sizes[b]) + int(r.integers(0, 3))
        return start, at + 1

    (start, slots), (out_start, out_slots) = places(ctx_len), places(kept)

    def cache(n):
        x = torch.randn(L, n, H, hd, generator=g).to(DTYPE[dtype])
        return x.transpose(1, 2).contiguous().cuda().transpose(1, 2) if layout == "heads" else x.cuda()

    k, v, k_out, v_out = cache(slots), cache(slots), cache(out_slots), cache(out_slots)
    mass = torch.from_numpy(mass_of(r, L, H, slots).astype(np.float32)).cuda()
    mass_out = torch.randn(L, H, out_slots, generator=g).cuda()
    want_k, want_v, want_m = k_out.clone(), v_out.clone(), mass_out.clone()
    m = mass.cpu().numpy()
    want = []
    for b in range(B):
        rows = [[_kept(m[l, h, start[b]:start[b] + ctx_len[b]], int(keep[b]), first, recent) for h in range(H)] for l in range(L)]
        want.append(np.array(rows, dtype=np.int32).reshape(L, H, -1))
        for l in range(L):
            for h in range(H):
                src, dst = int(start[b]) + torch.tensor(rows[l][h], dtype=torch.long), slice(int(out_start[b]), int(out_start[b]) + int(kept[b]))
                want_k[l, dst, h], want_v[l, dst, h], want_m[l, h, dst] = k[l, src, h], v[l, src, h], mass[l, h, src]
    if ctx is None:
        ctx = Context(device="cuda:0")
        ctx.reserve(evict_rows=int(kept.sum()), evict_utts=B, evict_heads=(L, H))
    got = ctx.kv_evict(k, v, mass, start, ctx_len, keep, first, recent, k_out, v_out, out_start, mass_out=mass_out if want_mass else None, want_rows=want_rows)
    torch.cuda.synchronize()
    if want_rows:
        assert np.array_equal(got.cpu().numpy(), np.concatenate(want, -1))
    assert torch.equal(k_out, want_k) and torch.equal(v_out, want_v)             # rows of nobody among them
    if want_mass:
        assert torch.equal(mass_out.view(torch.int32), want_m.view(torch.int32))


def _weights(r, *shape):
    return np.exp(2 * r.standard_normal(shape))


@pytest.mark.parametrize("dtype, hd", [("f16", 128), ("bf16", 64), ("f32", 64), ("f32", 4), ("f32", 36)])
@pytest.mark.parametrize("layout", ["slots", "heads"])
def test_ragged_batches(dtype, hd, layout):
    _check(_weights, dtype, hd=hd, ctx_len=(0, 1, 30, 64, 65, 200, 1030, 7), keep=(5, 5, 11, 63, 30, 200, 257, 5), first=2, recent=3, layout=layout)


@pytest.mark.parametrize("n, keep, first, recent", [(1, 0, 0, 0), (5, 0, 0, 0), (5, 1, 1, 0), (5, 1, 0, 1), (5, 4, 2, 2), (5, 5, 9, 9), (1024, 1023, 0, 0), (1025, 1, 0, 0),
                                                    (3000, 1500, 1, 1000), (70001, 9000, 16, 500), (70001, 69999, 0, 0), (140007, 20000, 0, 7)])
def test_lengths(n, keep, first, recent):
    _check(_weights, ctx_len=(n,), keep=(keep,), first=first, recent=recent, L=1, H=2)


@pytest.mark.parametrize("n", [50, 3000, 40000])
def test_equal_weights(n):
    """All alike; a few values; zeros of both signs."""
    _check(lambda r, *s: np.full(s, 0.25), ctx_len=(n,), keep=(n // 3,), L=1, first=1, recent=2)
    _check(lambda r, *s: r.integers(0, 3, size=s) / 7, ctx_len=(n,), keep=(n // 2,), L=1)
    _check(lambda r, *s: np.where(r.random(s) < 0.5, 0.0, -0.0), ctx_len=(n,), keep=(n // 2,), L=1)


@pytest.mark.parametrize("n", [60, 5000, 20000])
def test_weights_that_are_not_finite(n):
    values = np.array([np.nan, -np.nan, np.inf, -np.inf, 0.0, -1.5, 2.5, 1e-42, -1e-42, 3e38])
    for keep in (1, n // 4, n // 2, n - 5):
        _check(lambda r, *s: values[r.integers(0, len(values), size=s)], ctx_len=(n,), keep=(keep,), L=1, seed=keep)


def test_long_and_short_contexts_in_one_call():
    _check(_weights, ctx_len=(20000, 3, 8192, 8193, 0, 500, 40000), keep=(7000, 3, 1, 8000, 0, 100, 39990), first=1, recent=0, L=1, H=2)
    _check(lambda r, *s: r.integers(0, 2, size=s) / 3, ctx_len=(30000, 100, 9000), keep=(16000, 100, 4500), first=5, recent=3, L=2, H=1)


def test_contexts_of_more_chunks_than_pieces():
    """600000 rows: two chunks a piece; values that fill one bin of every digit, and ordinary ones."""
    _check(_weights, ctx_len=(600000,), keep=(150001,), first=3, recent=70000, L=1, H=1, hd=64)
    _check(lambda r, *s: np.full(s, 0.125), ctx_len=(600001,), keep=(300000,), L=1, H=1, hd=64)


def test_optional_outputs():
    _check(_weights, want_rows=False)
    _check(_weights, want_mass=False)
    _check(_weights, want_rows=False, want_mass=False, ctx_len=(33, 50), keep=(20, 50))


def test_all_layers_of_a_model():
    _check(_weights, L=24, H=8, hd=128, ctx_len=(211, 340), keep=(128, 128), first=4, recent=32)


def test_caches_beyond_four_gib():
    """64 K/V heads of 128 dims: 16 KB a row, rows behind 2^18 lie beyond 4 GiB in both caches."""
    n, far = 2 ** 18 + 600, 300
    k = torch.zeros(1, n, 64, 128, dtype=torch.float16, device="cuda")
    k[:, -far:] = torch.randn(far, 64, 128, device="cuda").half()
    mass = torch.ones(1, 64, n, device="cuda")
    mass[:, :, -far::3] = 2.0
    k_out = torch.zeros_like(k)
    ctx = Context(device="cuda:0")
    keep = len(range(n - far, n, 3))
    ctx.reserve(evict_rows=keep, evict_utts=1, evict_heads=(1, 64))
    ctx.kv_evict(k, k, mass, [n - 500], [500], [keep], 0, 0, k_out[:, ::1], k_out.clone(), [n - 200])
    assert torch.equal(k_out[:, n - 200:n - 200 + keep], k[:, -far::3])


def test_captured_calls():
    r = np.random.default_rng(4)
    s = torch.cuda.Stream()
    B = 400                                                  # more than the arguments of one launch hold
    n, keep = r.integers(1, 60, size=B), np.full(B, 20)
    kept = np.minimum(n, keep)
    start, out_start = np.cumsum(n) - n, np.cumsum(kept) - kept
    with torch.cuda.stream(s):
        k, v = torch.randn(2, 1, int(n.sum()), 2, 64, device="cuda").half()
        mass = torch.rand(1, 2, int(n.sum()), device="cuda")
        ctx = Context(device="cuda:0", stream=s)
        ctx.reserve(evict_rows=int(kept.sum()), evict_utts=B, evict_heads=(1, 2))
        a, b = (torch.zeros(1, int(kept.sum()), 2, 64, dtype=torch.float16, device="cuda") for _ in range(2))
        ctx.kv_evict(k, v, mass, start, n, keep, 1, 2, a, b, out_start)
        want = a.clone(), b.clone()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ctx.kv_evict(k, v, mass, start, n, keep, 1, 2, a, b, out_start)
        c, d = torch.zeros_like(a), torch.zeros_like(a)
        for _ in range(3):
            a.zero_()
            b.zero_()
            ctx.kv_evict(k, v, mass, start[::-1], n[::-1], keep, 0, 0, c, d, out_start[::-1])
            s.synchronize()
            graph.replay()
            s.synchronize()
            assert torch.equal(a, want[0]) and torch.equal(b, want[1])
