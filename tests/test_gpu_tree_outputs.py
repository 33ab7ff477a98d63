"""Where tree_attention and verify_tree write: outputs that lie between other data of the caller, fp32 rows that end inside a vector of the kernels."""
import numpy as np
import pytest
import torch

from paper_2603_11243_amd.binding import Context
from tests import test_gpu_verify_tree as rounds
from tests.test_gpu_tree_attention import Call, _batch
from workloads.configs import ModelCfg

pytestmark = pytest.mark.gpu

HEADS_32 = [(4, 2, 68), (2, 2, 76), (6, 2, 100), (3, 1, 124), (4, 4, 60)]
HEADS_16 = [(4, 2, 64), (16, 8, 128)]
ALL = [("f32", h) for h in HEADS_32] + [(d, h) for d in ("f16", "bf16") for h in HEADS_16]
GUARD = 64                                                   # values before and behind an output: a multiple of 16 bytes


def _guarded(shape, dtype):
    n = int(np.prod(shape))
    whole = torch.full((n + 2 * GUARD,), 12345.0, dtype=dtype, device="cuda")
    return whole, whole[GUARD:GUARD + n].view(shape)


def _check_guarded(call):
    whole, out = _guarded(call.q.shape, call.dtype)
    whole_lse, call.lse = _guarded(call.lse.shape, torch.float32)
    call.check(out=out)
    for x in (whole, whole_lse):
        assert (x[:GUARD] == x[0]).all() and (x[-GUARD:] == x[0]).all() and x[0] == torch.tensor(12345.0, dtype=x.dtype, device="cuda")
    return out.clone()


@pytest.mark.parametrize("dtype, heads", ALL)
def test_ragged_batches_write_their_rows_alone(dtype, heads):
    """Tiles of 16 rows and of more, whole contexts: every output element has one value, run after run, and nothing around them changes."""
    for nodes in ([1, 1, 2, 3], [7, 16, 9, 40]):
        c = Call(dtype, heads, [0, 5, 33, 129], _batch(41, None, nodes), seed=42)
        first = _check_guarded(c)
        assert torch.equal(_check_guarded(c), first)


@pytest.mark.parametrize("dtype, heads", ALL)
@pytest.mark.parametrize("nodes", [1, 6, 20])
def test_cut_contexts_write_their_rows_alone(dtype, heads, nodes):
    _check_guarded(Call(dtype, heads, [5003, 17], _batch(43, None, [nodes, 2]), seed=44))


@pytest.mark.parametrize("head_dim", [68, 100, 124])
def test_rounds_of_fp32_models_of_any_head_dim(head_dim, monkeypatch):
    cfg = ModelCfg(n_layers=2, d_model=96, n_q_heads=4, n_kv_heads=2, head_dim=head_dim, d_ff=128, vocab=512, dtype="f32")
    monkeypatch.setitem(rounds.MODELS, "f32_any", (cfg, "f16"))
    rounds.test_rounds("f32_any", [40, 3, 100, 64], [9, 1, 20, 16])


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_eviction_between_caches_of_any_order(dtype):
    """Slots outside with the layers inside them, heads outside, layers outside: the rows that caches of the usual order get, and nothing around them."""
    L, H, hd, n, keep = 3, 2, 64, [70, 33], [20, 9]
    g = torch.Generator().manual_seed(45)
    k, v = (torch.randn(L, 110, H, hd, generator=g).to(dtype).cuda() for _ in range(2))
    mass = torch.rand(L, H, 110, generator=g).cuda()
    ctx = Context(device="cuda:0")
    ctx.reserve(evict_rows=sum(keep), evict_utts=2, evict_heads=(L, H))
    results = []
    for order in ((0, 1, 2), (1, 0, 2), (2, 0, 1), (2, 1, 0)):
        back = [order.index(i) for i in range(3)] + [3]
        lay = lambda x: x.permute(*order, 3).contiguous().permute(back)
        k_out, v_out = (lay(torch.full((L, 40, H, hd), 7.0, dtype=dtype, device="cuda")) for _ in range(2))
        rows = ctx.kv_evict(lay(k), lay(v), mass, [0, 75], n, keep, 3, 5, k_out, v_out, [4, 28], want_rows=True)
        torch.cuda.synchronize()
        results.append((rows, k_out.clone(), v_out.clone()))
    for r in results[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, results[0]))
    left = torch.ones(40, dtype=torch.bool)
    left[4:24] = left[28:37] = False
    assert (results[0][1][:, left.cuda()] == 7).all() and not (results[0][1][:, ~left.cuda()] == 7).all(-1).any()
    ctx.close()
