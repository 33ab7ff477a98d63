"""tree_attention, tree_path, kv_evict, verify_tree and accept_tree refuse bad arguments on the host (no GPU: no pointer is followed)."""
import ctypes as C
import os

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, ESHAPE, EWORKSPACE, EUNSUPPORTED = -1, -2, -3, -5
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(os.path.join(ROOT, "paper_2603_11243_amd", "libssd.so")):
        from paper_2603_11243_amd.build import build_library
        build_library(verbose=False)
    from paper_2603_11243_amd import binding
    return binding.load_library()


@pytest.fixture()
def ctx(lib):
    h = C.c_void_p()
    assert lib.ssd_create(C.byref(h), None, None, None) == 0
    yield h
    lib.ssd_destroy(h)


def i32(a):
    return np.asarray(a, dtype=np.int32)


def view(base=1 << 40, slots=100, ss=256, hs=128, ls=0, L=1, H=2, hd=128, dtype=F16, k=None, v=None):
    from paper_2603_11243_amd.binding import KvViewC
    return KvViewC(base if k is None else k, base + (1 << 30) if v is None else v, slots, ss, hs, ls, L, H, hd, dtype)


P = C.c_void_p(1 << 20)
p = lambda a: None if a is None else a.ctypes.data


Q = C.c_void_p(1 << 24)


def attention(lib, ctx, kv=None, q=Q, q_stride=512, hq=4, B=2, start=i32([0, 50]), n=i32([20, 30]), cu=i32([0, 3, 5]), parent=i32([-1, 0, 0, -1, -1]), scale=0.1,
              out=P, lse=None, mass=None):
    return lib.tree_attention(ctx, q, q_stride, hq, C.byref(view() if kv is None else kv), B, p(start), p(n), p(cu), p(parent), C.c_float(scale), out, lse, mass)


def test_attention(lib, ctx):
    call = lambda **k: attention(lib, ctx, **k)
    assert call() == EWORKSPACE and b"tree_attention" in lib.ssd_last_error(ctx)
    for k in ({"q": None}, {"out": None}, {"start": None}, {"n": None}, {"cu": None}, {"parent": None}, {"B": 0}, {"B": -3}):
        assert call(**k) == EINVAL, k
    assert lib.tree_attention(None, P, 512, 4, C.byref(view()), 1, p(i32([0])), p(i32([1])), p(i32([0, 1])), p(i32([-1])), C.c_float(1), P, None, None) == EINVAL
    assert lib.tree_attention(ctx, P, 512, 4, None, 1, p(i32([0])), p(i32([1])), p(i32([0, 1])), p(i32([-1])), C.c_float(1), P, None, None) == EINVAL
    assert call(cu=i32([1, 3, 5])) == EINVAL and call(cu=i32([0, 3, 2])) == EINVAL
    for parent in ([0, 0, 0, -1, -1], [-1, 1, 0, -1, -1], [-1, 0, -2, -1, -1], [-1, 0, 0, 2, -1], [-1, 0, 0, -1, 1 << 30]):
        assert call(parent=i32(parent)) == EINVAL
    assert call(start=i32([-1, 50])) == EINVAL and call(n=i32([20, -1])) == EINVAL
    assert call(start=i32([0, 69])) == EINVAL                   # 30 rows and 2 nodes from slot 69: one too many
    assert call(start=i32([0, 68])) == EWORKSPACE
    assert call(start=i32([0, 22])) == EWORKSPACE and call(start=i32([0, 22]), mass=P) == EINVAL      # shared slots, with weights
    assert call(start=i32([2 ** 31 - 5, 50])) == EINVAL
    for bad in (float("nan"), float("inf")):
        assert call(scale=bad) == EINVAL
    assert call(hq=3) == ESHAPE and call(hq=0) == ESHAPE
    assert call(q_stride=511) == EINVAL and call(q_stride=516) == EINVAL and call(q=C.c_void_p(8)) == EINVAL and call(out=C.c_void_p(8)) == EINVAL
    assert call(kv=view(L=2, ls=25600)) == EINVAL
    near = lambda n: C.c_void_p((1 << 24) + n)
    assert call(out=near(0)) == EINVAL and call(out=near(5120 - 16)) == EINVAL and call(out=near(5120)) == EWORKSPACE and call(out=near(-5120 + 16)) == EINVAL
    many = i32(np.arange(1025) - 1)
    assert call(B=1, cu=i32([0, 1025]), parent=many, kv=view(slots=5000), n=i32([20])) == ESHAPE
    assert call(B=1, cu=i32([0, 1024]), parent=many, kv=view(slots=5000), n=i32([20])) == EWORKSPACE
    # nothing to do is not an error
    assert call(cu=i32([0, 0, 0]), q=None, out=None) == 0


def test_views(lib, ctx):
    call = lambda **k: attention(lib, ctx, kv=view(**k), hq=4, q_stride=1024)
    for good in ({}, {"hd": 64, "hs": 64}, {"dtype": BF16}, {"dtype": F32, "hd": 36, "hs": 36, "ss": 72}, {"ss": 128, "hs": 12800}, {"ss": 128, "hs": 20000},
                 {"H": 1, "ss": 128, "hs": 0}):
        assert call(**good) == EWORKSPACE, (good, lib.ssd_last_error(ctx))
    for bad in ({"k": 0}, {"v": 0}, {"k": 8}, {"v": 24}, {"slots": 0}, {"slots": (1 << 30) + 1}, {"slots": 1 << 31}, {"H": 0}, {"hd": 0}, {"L": 0}, {"ss": 264, "hs": 132}, {"ss": 260},
                {"ss": 192}, {"hs": 64}, {"hs": -128}, {"ss": -256}, {"ss": 0}, {"ss": 128, "hs": 12792}, {"ss": 128, "hs": 256}):
        assert call(**bad) == EINVAL, bad
    assert call(dtype=3) == EUNSUPPORTED
    for bad in ({"hd": 32}, {"hd": 96}, {"hd": 256, "hs": 256, "ss": 512}, {"dtype": F32, "hd": 6, "hs": 8}, {"dtype": F32, "hd": 132, "hs": 132, "ss": 264}, {"ss": 1 << 24}):
        assert call(**bad) == ESHAPE, bad


def test_path(lib, ctx):
    def call(logp=P, B=1, cu=i32([0, 3]), parent=i32([-1, 0, 0]), tau=0.1, a=P, b=P, c=P):
        return lib.tree_path(ctx, logp, B, p(cu), p(parent), C.c_float(tau), a, b, c)
    assert call() == EWORKSPACE
    for k in ({"logp": None}, {"a": None}, {"b": None}, {"c": None}, {"cu": None}, {"parent": None}, {"B": 0}, {"tau": float("nan")}, {"parent": i32([0, 0, 0])}):
        assert call(**k) == EINVAL, k
    assert call(cu=i32([0, 1025]), parent=i32(np.arange(1025) - 1)) == ESHAPE
    assert lib.ssd_tree_workspace_bytes(ctx, 0, 0, 0, -1, 1) == 0 and lib.ssd_tree_workspace_bytes(None, 0, 0, 0, 1, 1) == 0


def test_evict(lib, ctx):
    far = 1 << 44

    def call(kv=None, mass=P, B=2, start=i32([0, 50]), n=i32([40, 30]), keep=i32([10, 20]), first=2, recent=3, to=None, out=i32([0, 10]), mass_out=None, rows=None):
        return lib.kv_evict(ctx, C.byref(view() if kv is None else kv), mass, B, p(start), p(n), p(keep), first, recent,
                            C.byref(view(base=far, slots=30) if to is None else to), p(out), mass_out, rows)
    assert call() == EWORKSPACE
    for k in ({"mass": None}, {"start": None}, {"n": None}, {"keep": None}, {"out": None}, {"B": 0}, {"first": -1}, {"recent": -1}, {"keep": i32([-1, 20])},
              {"keep": i32([4, 20])}, {"out": i32([0, 11])}, {"out": i32([0, 9])}, {"out": i32([-1, 10])}, {"start": i32([61, 50])}, {"n": i32([40, 51])}):
        assert call(**k) == EINVAL, k
    assert call(keep=i32([10, 20]), first=1 << 30, recent=1 << 30) == EINVAL
    assert call(keep=i32([40, 30]), first=99, recent=99, to=view(base=far, slots=70), out=i32([0, 40])) == EWORKSPACE      # nothing goes
    for to in (view(base=far, hd=64, hs=64, slots=30), view(base=far, dtype=BF16, slots=30), view(base=far, H=1, slots=30), view(base=far, L=2, ls=7680, slots=30),
               view(base=far, slots=30, v=far), view(slots=30), view(base=far, slots=30, v=(1 << 40) + 100 * 512 - 16), view(base=far, slots=30, k=(1 << 40) + (1 << 30) - 30 * 512 + 16)):
        assert call(to=to) == EINVAL
    assert call(mass=P, mass_out=C.c_void_p((1 << 20) + 796)) == EINVAL and call(mass=P, mass_out=C.c_void_p((1 << 20) + 800)) == EWORKSPACE
    assert call(keep=i32([0, 0]), first=0, recent=0) == 0                        # nothing stays: nothing to copy
    many = 65536
    assert call(B=many, start=i32([0] * many), n=i32([0] * many), keep=i32([0] * many), out=i32([0] * many), first=0, recent=0) == ESHAPE
    many, to = 2100, view(base=1 << 45, slots=1 << 25)                           # more than 2^24 rows of overlapping contexts
    assert call(kv=view(slots=8192), B=many, start=i32([0] * many), n=i32([8192] * many), keep=i32([8192] * many), out=i32(np.arange(many) * 8192), to=to) == ESHAPE
    assert lib.ssd_evict_workspace_bytes(ctx, 0, 1, 1, 1) == 0 and lib.ssd_evict_workspace_bytes(ctx, 1, 1, 10, 1) > 40


def test_calls_that_need_a_model(lib, ctx):
    from paper_2603_11243_amd.binding import KvViewC
    cu, one = i32([0, 1]), i32([-1])
    v = KvViewC()
    assert lib.ssd_kv_cache_view(ctx, None, 0, C.byref(v)) == EINVAL and lib.ssd_kv_cache_view(None, None, 0, C.byref(v)) == EINVAL
    assert lib.verify_tree(ctx, P, 1, p(cu), p(one), p(i32([0])), p(i32([1])), None, None, P) == EINVAL
    assert lib.accept_tree(ctx, P, P, 1, p(cu), p(one), C.c_float(0.1), None, None, None, P, P, P, P, P) == EINVAL
    assert lib.ssd_verify_tree_workspace_bytes(ctx, 10, 1) == 0


def test_workspace_sizes_serve_smaller_calls(lib, ctx):
    last = 0
    for n in (1, 7, 63, 500, 5000):
        for B in (1, 3, 64):
            assert lib.ssd_tree_workspace_bytes(ctx, 16, 8, 128, n, B) >= lib.ssd_tree_workspace_bytes(ctx, 16, 8, 128, n, 1) >= last
            assert lib.ssd_tree_workspace_bytes(ctx, 16, 8, 128, n, B) >= lib.ssd_tree_workspace_bytes(ctx, 0, 0, 0, n, B)
        last = lib.ssd_tree_workspace_bytes(ctx, 16, 8, 128, n, 1)


def test_more_tiles_than_a_launch_has(lib, ctx):
    """512 query heads on one: 4096 tiles of 128 rows an utterance of 1024 nodes."""
    one = dict(kv=view(base=1 << 50, slots=1 << 20, H=1, ss=128, hs=0), hq=512, q_stride=1 << 16, q=C.c_void_p(1 << 45), out=C.c_void_p(1 << 46))
    for B, want in ((15, EWORKSPACE), (16, ESHAPE), (800, ESHAPE)):
        assert attention(lib, ctx, B=B, start=i32(np.arange(B) * 1024), n=i32([0] * B), cu=i32(np.arange(B + 1) * 1024), parent=i32(np.tile(np.arange(1024) - 1, B)),
                         **one) == want


def test_host_memory_that_does_not_suffice_is_an_error():
    """In a process of its own, whose address space may not grow by what the call builds."""
    import subprocess
    import sys
    code = """
import ctypes as C, resource, sys
import numpy as np
sys.path[:0] = [%r, %r]
from test_tree_abi_host import attention, i32, view
from paper_2603_11243_amd import binding
lib, h = binding.load_library(), C.c_void_p()
assert lib.ssd_create(C.byref(h), None, None, None) == 0
B = 8000
args = dict(kv=view(base=1 << 50, slots=1 << 23, H=1, ss=128, hs=0), hq=1, q_stride=128, q=C.c_void_p(1 << 45), out=C.c_void_p(1 << 46), B=B, start=i32(np.arange(B) * 1024),
            n=i32([0] * B), cu=i32(np.arange(B + 1) * 1024), parent=i32(np.tile(np.arange(1024) - 1, B)))
assert attention(lib, h, **args) == -3
now = int(open('/proc/self/statm').read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (now + (8 << 20), resource.getrlimit(resource.RLIMIT_AS)[1]))
rc = attention(lib, h, **args)
assert rc == -2 and b'tree_attention' in lib.ssd_last_error(h), rc
print('refused')
""" % (ROOT, os.path.join(ROOT, "tests"))
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert run.returncode == 0 and "refused" in run.stdout, run.stderr[-2000:]
