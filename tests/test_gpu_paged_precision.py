"""Weights and log-sum-exps of paged_attention keep fp32's precision: cases in which what a weight lost is what is left."""
import numpy as np
import pytest
import torch

from pages import Pool
from test_gpu_paged_attention import PAIRS, _context, _queries

FP32 = [("f32", "f32"), ("f32", "e4m3"), ("f32", "i8")]


def _parts(pool, b):
    """Keys and values [heads, rows, head_dim] of utterance b in 64 bits."""
    return (pool.rows(pool.value(name), b)[0].transpose(1, 0, 2) for name in ("k", "v"))


def _dot(q, pool, b, h, c):
    """Scores of the rows of utterance b for query head h, and how far off they may be: c values of 16 bits a query, c head_dim products added in fp32, and scales."""
    x, scale = q[b, 0, h].double().cpu().numpy(), pool.hd ** -0.5
    k = list(_parts(pool, b))[0][h * pool.H // q.shape[2]]
    return k @ x * scale, (c * pool.hd + 8) * 2.0 ** -24 * scale * (abs(k) @ abs(x)).max()


def _in_pairs(pool):
    """The values of every odd row are those of the row before it with the other sign."""
    for b, n in enumerate(pool.ctx_host):
        for j in range(1, n, 2):
            page, at, one = int(pool.table_host[b, j // pool.page_rows]), j % pool.page_rows, (j - 1) % pool.page_rows
            v = pool.parts["v"]
            v[0, page, :, at] = (-v[0, page, :, one].float()).to(v.dtype)
            if "v_scale" in pool.parts:
                pool.parts["v_scale"][0, page, :, at] = pool.parts["v_scale"][0, page, :, one]


def _two_values(w):
    """The part of weights that two bfloat16 values hold."""
    top = torch.from_numpy(w).float().bfloat16().double()
    return (top + (torch.from_numpy(w) - top).float().bfloat16().double()).numpy()


def _biased(s):
    """Weights 2^s as 2^(s - 32) with the exponent rounded to fp32."""
    return 2.0 ** ((s - 32).astype(np.float32).astype(np.float64) + 32)


def _errors(weights):
    """Of two rows of values 1 and -1: how far (w0 - w1) / (w0 + w1) of the weights of some scores (to base 2, at most 0) is off, in units of the test's bound on them."""
    s = -np.random.default_rng(0).uniform(0, 2e-3, 1000)
    true, got = 2.0 ** s, weights(s)
    return abs((1 - got) / (1 + got) - (1 - true) / (1 + true)) / (2.0 ** -22 + 2e-7)


def test_the_bound_tells_what_a_weight_lost():
    """Weights of two 16-bit values, and of exponents with a bias, are further off than the tests below allow; ones rounded to fp32 are not."""
    assert _errors(lambda s: _two_values(2.0 ** s)).max() > 4 and _errors(_biased).max() > 1.3
    assert _errors(lambda s: (2.0 ** s).astype(np.float32).astype(np.float64)).max() < 0.2


@pytest.mark.gpu
@pytest.mark.parametrize("pair", FP32)
@pytest.mark.parametrize("n", [2, 4])
@pytest.mark.parametrize("hd, n_new", [(64, 1), (128, 1), (64, 17)])
def test_what_is_left_of_values_that_cancel(pair, n, hd, n_new):
    """Two rows, or four, whose values are the same but for the sign, and nearly the same scores: the output is the difference of their weights.  A weight is off by the
    exponential's 2^-23 and twice its score's error (its own and the maximum's); the largest is 1.  Sums of a pair are exact but for what is left, a rounding of a
    sum with the next pair is 2^-24 of one value of four: together less than 2^-22 of the mean magnitude; every other rounding, some ten, is relative to the output."""
    heads, B = (2, 2, hd), 64
    pool, q = Pool(pair[1], heads[1:], [n + n_new - 1] * B, 16), _queries("f32", B, n_new, heads, scale=1e-3)
    _in_pairs(pool)
    out = _context(B, n_new, heads, 64).paged_attention(q, pool.pages(), pool.table, pool.ctx_len).double().cpu().numpy()
    worst = 0.0
    for b in range(B):
        v = list(_parts(pool, b))[1]
        for h in range(2):
            s, d = _dot(q, pool, b, h, 3)
            p = np.exp(s[:n] - s[:n].max())
            p /= p.sum()
            want = p @ v[h, :n]
            tol = (2.0 ** -22 + 2 * d) * (p @ abs(v[h, :n])) + 2.0 ** -20 * abs(want) + 2.0 ** -100
            worst = max(worst, (abs(out[b, 0, h] - want) / tol).max())
    assert worst <= 1, worst


@pytest.mark.gpu
@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("n", [1, 2])
def test_log_sum_exp_of_a_row_or_two(pair, n):
    """Of one row it is its score: off by the score's error, the factors to base 2 and back and the products with them (2^-22 of it).  Of two, a logarithm near 1 and a sum more."""
    heads, B = (4, 2, 64), 64
    pool, q = Pool(pair[1], heads[1:], [n] * B, 16), _queries(pair[0], B, 1, heads, scale=1e-3)
    lse = torch.empty(B, 1, 4, device="cuda")
    _context(B, 1, heads, 16).paged_attention(q, pool.pages(), pool.table, pool.ctx_len, lse=lse)
    got = lse.double().cpu().numpy()
    for b in range(B):
        for h in range(4):
            s, d = _dot(q, pool, b, h, 3)
            want = np.log(np.exp(s).sum())
            assert abs(got[b, 0, h] - want) <= d + 2.0 ** -22 * abs(want) + (n - 1) * 2.0 ** -22, (b, h)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("n, n_new", [(40, 1), (40, 9), (5000, 2)])
def test_half_outputs_beyond_half(kind, n, n_new):
    """Means of values beyond half are stored as its largest ones, and the flag says so; where only the values are beyond it nothing is clamped or raised.  A wavefront adds at most 64 times 32 products, each off by
    2^-24, of weights off by 2^-17: 1.3e-4 of a value, less than what lies between 65504 or 65508 and where half's rounding goes elsewhere."""
    heads = (4, 2, 64)
    pool, q = Pool(kind, heads[1:], [n], 16), _queries("f16", 1, n_new, heads)
    c = _context(1, n_new, heads, n + 16)
    v, scale = pool.parts["v"].view(torch.uint8), pool.parts["v_scale"]
    one = torch.tensor([1.0]).to(pool.parts["v"].dtype).view(torch.uint8).item()
    run = lambda: c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len)

    def fill(x):
        v.fill_(one)
        scale.copy_(torch.where(scale.isnan(), scale, x))

    fill(65504.0)
    c.device_flags()
    assert (run() == 65504).all() and c.device_flags() == 0
    fill(-65508.0)
    assert (run() == -65504).all() and c.device_flags() == 0
    fill(70000.0)
    assert (run() == 65504).all() and c.device_flags() == 2
    fill(-1e30)
    assert (run() == -65504).all() and c.device_flags() == 2
    fill(float("inf"))
    assert not torch.isfinite(run()).any() and c.device_flags() == 2
    fill(1e5)                                                # every other row of the other sign, the queries too small to tell them apart
    _in_pairs(pool)
    q.mul_(1e-4)
    out = run()
    assert torch.isfinite(out).all() and (out.abs() < 65504).all() and c.device_flags() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n", [40, 5000])
def test_infinities_of_half_pages_stay(n):
    heads = (4, 2, 64)
    pool, q = Pool("f16", heads[1:], [n], 16), _queries("f16", 1, 1, heads)
    pool.parts["v"].fill_(65504.0)
    c = _context(1, 1, heads, n + 16)
    c.device_flags()
    assert (c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len) == 65504).all()
    pool.parts["v"].fill_(float("inf"))
    assert not torch.isfinite(c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len)).any() and c.device_flags() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("pair", [p for p in PAIRS if p[0] != "f16"])
def test_small_values(pair):
    """Values times a power of two: outputs times the same, down to where bits are lost (8-bit rows below 2^-66, others below 2^-90).  A part of a weight is held to
    2^-134 at worst (half of bfloat16's smallest step) where the largest is 2^-32 times the row's scale, 2^-75 or more: n 2^-27 of the largest value."""
    heads, n = (4, 2, 64), 300
    pool, q = Pool(pair[1], heads[1:], [n, 50], 16), _queries(pair[0], 2, 1, heads)
    c = _context(2, 1, heads, 320)
    run = lambda: c.paged_attention(q, pool.pages(), pool.table, pool.ctx_len).double()
    want, eight = run(), "v_scale" in pool.parts
    top = [max(pool.rows(pool.value("v"), b)[0].max(), -pool.rows(pool.value("v"), b)[0].min()) for b in range(2)]
    least = min(abs(pool.rows(pool.value("v"), b)[0]).max(-1).min() for b in range(2))
    down = int(np.log2(least) + 66) if eight else 80
    t = pool.parts["v_scale" if eight else "v"]
    t.copy_((t.double() * 2.0 ** -down).to(t.dtype))
    got = run() * 2.0 ** down
    u = torch.finfo(q.dtype).eps
    for b in range(2):
        assert ((got[b] - want[b]).abs() <= n * 2.0 ** -27 * top[b] + u * want[b].abs()).all(), (pair, down)
