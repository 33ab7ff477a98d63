"""tree_attention: bits of the weights that multiply the values, and values at the ends of the number range."""
import numpy as np
import pytest
import torch

from tests.test_gpu_tree_attention import Call, _batch
from trees import cu, sees

pytestmark = pytest.mark.gpu

HEADS_16 = [(16, 8, 128), (24, 8, 128), (4, 4, 64), (14, 2, 64)]
# A weight in two pieces of u relative error each: u^2.  IEEE half holds it with 2^11 at the row's largest, so that half a step below its normal numbers, 2^-25,
# is 2^-36 of that.
PIECES = {"f16": 2.0 ** -22, "bf16": 2.0 ** -16, "f32": 0.0}
LOW = {"f16": 2.0 ** -36, "bf16": 0.0, "f32": 0.0}


def _exact(call, scale):
    """out and its error bound as Call.exact derives them, with u^2 for the roundings of the weights in the place of u."""
    hq, hkv, hd = call.heads
    name = {torch.float16: "f16", torch.bfloat16: "bf16", torch.float32: "f32"}[call.dtype]
    u = torch.finfo(call.dtype).eps / 2
    q, k, v = (x.double().cpu().numpy() for x in (call.q, call.k, call.v))
    out, tol = np.zeros_like(q), np.zeros_like(q)
    node0 = cu(call.trees)
    for b, t in enumerate(call.trees):
        n, N, s0 = int(call.ctx_len[b]), len(t), int(call.kv_start[b])
        seen = np.concatenate([np.ones((N, n), bool), sees(t)], 1)
        for h in range(hq):
            kv, at = h * hkv // hq, (slice(node0[b], node0[b] + N), h)
            kk, vv, qq = k[s0:s0 + n + N, kv], v[s0:s0 + n + N, kv], q[at]
            vv = np.where(np.isfinite(vv), vv, 0)
            s = np.where(seen, qq @ kk.T * scale, -np.inf)
            d = ((hd + 4) * 2.0 ** -24 * abs(scale) * (abs(qq) @ abs(kk).T) * seen).max(1, initial=0)[:, None] + 2.0 ** -22
            p = np.exp(s - s.max(1, keepdims=True, initial=-np.inf))
            l = p.sum(1, keepdims=True)
            p /= l
            out[at] = p @ vv
            tol[at] = u * abs(out[at]) + (PIECES[name] + 2 * d + (n + N + 32) * 2.0 ** -24) * (p @ abs(vv)) + LOW[name] * (seen @ abs(vv)) / l
    return out, tol


def _check(call, **more):
    got = call.run(**more).double().cpu().numpy()
    out, tol = _exact(call, more.get("scale", call.heads[2] ** -0.5))
    assert np.isfinite(got).all()
    assert (abs(got - out) <= tol).all(), (abs(got - out) / tol).max()
    return got


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads", HEADS_16)
@pytest.mark.parametrize("nodes", [[1, 3, 2, 4], [9, 20, 7, 33], [70, 40, 100, 3]])
def test_weights_keep_more_bits_than_the_output(dtype, heads, nodes):
    """Outputs near zero are sums of larger terms of both signs: weights of the type's own bits would show there.  Whole and cut contexts."""
    _check(Call(dtype, heads, [60, 400, 0, 131], _batch(51, None, nodes), seed=52), mass=False)
    _check(Call(dtype, heads, [6000, 33, 700, 5], _batch(53, None, nodes), seed=54), mass=False)


@pytest.mark.parametrize("rows", [127, 4095, 60000])
@pytest.mark.parametrize("nodes", [1, 40])
def test_many_small_weights_of_one_size(rows, nodes):
    """A key with the value 0 in 32, and between them keys whose weights are 2^-26.4 of its own: what each loses is lost the same way, and must be little of it."""
    c = Call("f16", (2, 1, 128), [rows], [[-1] * nodes], seed=55)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.k.zero_()
    c.v[:] = 1024.0
    large = int(c.kv_start[0]) + torch.arange(0, rows, 32, device="cuda")
    c.k[large, 0, 0], c.v[large] = 26.4 * np.log(2.0), 0.0
    _check(c, mass=False, scale=1.0)


@pytest.mark.parametrize("dtype, heads", [("f16", (4, 2, 128)), ("bf16", (4, 2, 128)), ("f16", (16, 4, 64)), ("bf16", (6, 2, 64)), ("f32", (4, 2, 64)), ("f32", (2, 2, 100))])
@pytest.mark.parametrize("ctx_len, nodes", [([40, 300], [1, 6]), ([7, 260], [12, 40]), ([5003, 2000], [2, 20])])
def test_an_infinite_value_is_the_output_of_its_column(dtype, heads, ctx_len, nodes):
    """Seen infinities in cached rows (whole blocks, the block of the nodes) and in a node; rows that do not see the node, and other columns, keep their results."""
    c = Call(dtype, heads, ctx_len, _batch(56, None, nodes, ("random",)), seed=57)
    want, tol = _exact(c, heads[2] ** -0.5)
    at = cu(c.trees)
    column = 0
    for b, t in enumerate(c.trees):
        group = heads[0] // heads[1]
        n, s0 = int(c.ctx_len[b]), int(c.kv_start[b])
        for row in (0, n // 2, n - 1, n + len(t) // 2):
            for kv in range(heads[1]):
                column = (column + 7) % heads[2]
                bad = float("inf") if column % 2 else float("-inf")
                c.v[s0 + row, kv, column] = bad
                who = np.ones(len(t), bool) if row < n else sees(t)[:, row - n]
                rows = at[b] + np.nonzero(who)[0]
                for h in range(kv * group, (kv + 1) * group):
                    old = want[rows, h, column]
                    want[rows, h, column] = np.where(np.isinf(old) & (old != bad), np.nan, bad)
    got = c.run(mass=False).double().cpu().numpy()
    odd = ~np.isfinite(want)
    assert np.array_equal(got[odd], want[odd], equal_nan=True)
    # (columns that hold an infinity elsewhere: _exact took it into account where it is seen, the rest is as before)
    assert (abs(got[~odd] - want[~odd]) <= tol[~odd]).all()


def _alike(dtype, heads, ctx_len, trees, seed):
    """Every key counts the same."""
    c = Call(dtype, heads, ctx_len, trees, seed=seed)
    c.q.zero_()
    return c


ENDS = [("bf16", (16, 8, 128)), ("bf16", (4, 2, 64)), ("f32", (4, 2, 64)), ("f32", (2, 2, 100)), ("f16", (4, 2, 128))]


@pytest.mark.parametrize("dtype, heads", ENDS)
@pytest.mark.parametrize("ctx_len, nodes", [([300, 700], [1, 6]), ([515, 40], [40, 3]), ([900, 2], [3, 100]), ([20000, 30], [2, 5]), ([9000, 3000], [40, 70])])
@pytest.mark.parametrize("signs", ["one", "both"])
def test_means_of_values_near_the_end_of_the_range(dtype, heads, ctx_len, nodes, signs):
    """Sums of many of them are beyond fp32's range, their means are not."""
    c = _alike(dtype, heads, ctx_len, _batch(58, None, nodes, ("random", "chain")), 58)
    size = torch.rand(c.v.shape, generator=torch.Generator().manual_seed(59)).cuda() * 0.05 + 0.9
    if signs == "both":
        size *= torch.sign(torch.randn(c.v.shape, generator=torch.Generator().manual_seed(60)).cuda())
    c.v[:] = (size * torch.finfo(c.dtype).max).to(c.dtype)
    _check(c, mass=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at_the_end", [0.94, float("inf"), float("nan")])
def test_small_values_beside_rows_near_the_end_of_the_range(dtype, at_the_end):
    """Rows that see values near the end of the range, or infinities, beside rows that see small ones: the latter notice nothing."""
    left, right = 600, 5
    parent = [-1] + list(range(left - 1)) + [-1] + list(range(left, left + right - 1))
    c = _alike(dtype, (2, 1, 128), [40], [parent], 61)
    c.v[:] = (c.v.float() * 2.0 ** -110).to(c.dtype)
    first = int(c.kv_start[0]) + 40
    c.v[first:first + left] = 0
    want = c.run(mass=False)[left:].clone()
    out, tol = _exact(c, 1.0)
    assert (abs(want.double().cpu().numpy() - out[left:]) <= tol[left:]).all()
    c.v[first:first + left] = at_the_end * torch.finfo(c.dtype).max
    got = c.run(mass=False)
    assert torch.equal(got[left:], want)
    if at_the_end < 1:
        assert torch.isfinite(got).all() and (got[left - 1].float() > 0.8 * torch.finfo(c.dtype).max).all()
