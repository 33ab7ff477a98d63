"""Refusals of calls on trees that need a model."""
import pytest
import torch

from tests import test_gpu_verify_tree as rounds
from workloads.configs import ModelCfg

pytestmark = pytest.mark.gpu


def test_more_query_heads_than_a_tile_can_number(monkeypatch):
    """As tree_attention: at most 512 of them share a K/V head."""
    from paper_2603_11243_amd.binding import SsdError
    for heads, fits in ((512, True), (516, False)):
        cfg = ModelCfg(n_layers=1, d_model=32, n_q_heads=heads, n_kv_heads=1, head_dim=4, d_ff=64, vocab=512, dtype="f32")
        monkeypatch.setitem(rounds.MODELS, "many_heads", (cfg, "f16"))
        ctx, m, w, start, r = rounds._prefilled("many_heads", [20], 10)
        ids = torch.zeros(2, dtype=torch.int32, device="cuda")
        if fits:
            assert torch.isfinite(ctx.verify_tree(ids, [0, 2], [-1, 0], start, [20])).all()
        else:
            with pytest.raises(SsdError, match="512") as e:
                ctx.verify_tree(ids, [0, 2], [-1, 0], start, [20])
            assert e.value.code == -2
        ctx.close()
