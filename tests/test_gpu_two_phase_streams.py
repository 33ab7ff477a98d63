"""The two-phase schedule called while another stream than its context's is the current one."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify_tree import _weights
from workloads import WORKLOADS, make_ctc_batch, make_ctc_to_llm_map, make_verify_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["resident", "offload"])
@pytest.mark.parametrize("trees", [None, dict(tau=0.5, depth=4)])
def test_another_stream_is_current(mode, trees):
    """The context's stream is busy when the calls are queued: results are read behind them all the same."""
    from paper_2603_11243_amd.binding import Context
    from paper_2603_11243_amd.pipeline import TwoPhaseDecoder
    wl = WORKLOADS["cfg1_tiny_f32"]
    cb, table = make_ctc_batch(wl), make_ctc_to_llm_map(wl)
    vi = make_verify_inputs(wl, cb.seconds, [np.zeros(0, np.int32)] * wl.B, device="cuda")
    runs, side = [], torch.cuda.Stream()
    for stream in (None, side):
        ctx = Context(wl.model, _weights(wl.model, 3), stream=stream)
        dec = TwoPhaseDecoder(ctx, wl, cb.logits.cuda(), cb.cu_frames, torch.from_numpy(table).cuda(), vi.speech_emb, vi.cu_speech,
                              torch.from_numpy(vi.prompt_ids).cuda(), vi.cu_prompt, budget=300, mode=mode, n_steps=9, trees=trees)
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(side):
                a = torch.randn(4096, 4096, device="cuda")
                for _ in range(100):                         # some tens of milliseconds
                    a = torch.matmul(a, a).clamp_(-1, 1)
        runs.append(dec.run(0.5))
        torch.cuda.synchronize()
        ctx.close()
    want, got = runs
    assert want["rejected"] > 0 and np.array_equal(got["accept_len"], want["accept_len"]) and set(got["tokens"]) == set(want["tokens"])
    assert all(np.array_equal(t, want["tokens"][b]) for b, t in got["tokens"].items())
