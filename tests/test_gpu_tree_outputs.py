"""Where tree_attention and verify_tree write: outputs that lie between other data of the caller, fp32 rows that end inside a vector of the kernels."""
import numpy as np
import pytest
import torch

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
