"""ssd_device_flags around captures, and of contexts without a model."""
import pytest
import torch

from pages import Pool
from paper_2603_11243_amd.binding import Context, SsdError
from workloads import WORKLOADS, make_model_weights

pytestmark = pytest.mark.gpu


def _move(kind="f16", n=5):
    """Pages, their table and lengths, rows for them: one utterance."""
    pool = Pool(kind, (2, 64), [n], 16)
    k, v = (torch.randn(n, 2, 64, device="cuda").half() for _ in range(2))
    return pool, (pool.pages(), pool.table, pool.ctx_len, k, v)


def test_before_calls_on_pages_a_context_without_a_model_answers_at_once():
    """0 without a wait, while its stream is captured too; the capture goes on."""
    side = torch.cuda.Stream()
    c, x, graph = Context(device="cuda:0", stream=side), torch.zeros(1000, device="cuda"), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        x.add_(1)
        assert c.device_flags() == 0
        x.add_(1)
    for i in range(3):
        graph.replay()
        side.synchronize()
        assert (x == 2 * i + 2).all() and c.device_flags() == 0
    c.close()


@pytest.mark.parametrize("model", [False, True])
def test_flags_are_refused_while_the_stream_is_captured(model):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        m = WORKLOADS["cfg1_tiny_f32"].model if model else None
        c = Context(m, make_model_weights(m, 1, device="cuda") if model else None, stream=side)
        pool, args = _move()
        c.kv_write_pages(*args)
        side.synchronize()
        x, graph = torch.zeros(1000, device="cuda"), torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            x.add_(1)
            with pytest.raises(SsdError, match="captured"):
                c.device_flags()
            c.kv_write_pages(*args)
            x.add_(1)
        pool.table.fill_(-1)                                 # what the replay finds
        for i in range(3):
            graph.replay()
            side.synchronize()
            assert (x == 2 * i + 2).all() and c.device_flags() == 4 and c.device_flags() == 0
    c.close()


@pytest.mark.parametrize("call", ["write", "read", "attention"])
def test_a_context_made_under_capture_has_flags(call):
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        pool, args = _move()
        q, out = (torch.randn(1, 4, 64, device="cuda").half() for _ in range(2))
        graph = torch.cuda.CUDAGraph()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            c = Context(device="cuda:0", stream=side)
            if call == "attention":
                c.paged_attention(q, *args[:3], out=out)
            else:
                (c.kv_write_pages if call == "write" else c.kv_read_pages)(*args)
        table = pool.table.clone()
        for bad in (0, 4, 0, 4):
            pool.table.copy_(table if not bad else torch.full_like(table, -1))
            graph.replay()
            assert c.device_flags() == bad
        c.close()
