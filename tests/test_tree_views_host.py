"""Caches whose slots, heads and layers lie inside each other in any order (no GPU: no pointer is followed)."""
import ctypes as C
import itertools

import numpy as np
import pytest

from test_tree_abi_host import EINVAL, EWORKSPACE, F32, P, ctx, i32, lib, p, view


def evict(lib, ctx, kv, to, rows=40, keep=10):
    start, n, k, out = i32([0]), i32([rows]), i32([keep]), i32([0])
    return lib.kv_evict(ctx, C.byref(kv), P, 1, p(start), p(n), p(k), 0, 0, C.byref(to), p(out), None, None)


@pytest.mark.parametrize("order", list(itertools.permutations("slh")))
@pytest.mark.parametrize("gap", [0, 8])
def test_any_order(lib, ctx, order, gap):
    """`order` from the innermost on, `gap` unused elements behind each row: accepted; an element less anywhere: rows that share memory."""
    hd, count = 128, {"s": 50, "l": 3, "h": 2}
    stride, inside = {}, hd + gap
    for d in order:
        stride[d] = inside
        inside *= count[d]
    kv = lambda **k: view(slots=50, L=3, H=2, hd=hd, **{**{"ss": stride["s"], "hs": stride["h"], "ls": stride["l"]}, **k})
    to = view(base=1 << 44, slots=20, L=3, H=2, ss=256, hs=128, ls=5120)
    assert evict(lib, ctx, kv(), to) == EWORKSPACE, lib.ssd_last_error(ctx)
    if gap:
        return
    for d, name in (("s", "ss"), ("h", "hs"), ("l", "ls")):
        assert evict(lib, ctx, kv(**{name: stride[d] - 8}), to) == EINVAL


def test_brute_force(lib, ctx):
    """Small views of every kind against the elements they name; strides that interleave rows of two dimensions are refused though no element is shared."""
    r = np.random.default_rng(1)
    agreed = 0
    for _ in range(3000):
        hd, n = 4, {"s": int(r.integers(1, 5)), "h": int(r.integers(1, 4)), "l": int(r.integers(1, 4))}
        st = {d: 4 * int(r.integers(1, 13)) for d in n}
        at = sorted(s * st["s"] + h * st["h"] + l * st["l"] + e for s in range(n["s"]) for h in range(n["h"]) for l in range(n["l"]) for e in range(hd))
        shares = len(set(at)) < len(at)
        kv = view(slots=n["s"], H=n["h"], L=n["l"], hd=hd, dtype=F32, ss=st["s"], hs=st["h"], ls=st["l"])
        to = view(base=1 << 44, slots=64, H=n["h"], L=n["l"], hd=hd, dtype=F32, ss=hd * n["h"], hs=hd, ls=64 * hd * n["h"])
        rc = evict(lib, ctx, kv, to, n["s"], 1)
        assert rc in (EINVAL, EWORKSPACE)
        if shares:
            assert rc == EINVAL, (n, st)
        agreed += rc == EWORKSPACE
    assert agreed > 300
