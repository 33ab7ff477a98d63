"""The two-phase schedule with the rows of rejected utterances in pages between the phases."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify import _tau_for
from tests.test_gpu_verify_tree import _weights
from workloads import WORKLOADS, make_ctc_batch, make_ctc_to_llm_map, make_model_weights, make_verify_inputs
from workloads.configs import scaled_down

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name, layers", [("cfg3_1b_ragged64", 2), ("cfg1_tiny_f32", 2)])
def test_rows_in_pages_between_the_phases(name, layers):
    """Pages of the cache's type: the tokens of the resident cache to the last one.  8 bits: the same decisions and first tokens (they are of the first phase), and a
    full continuation of every rejected utterance."""
    from paper_2603_11243_amd.binding import Context
    from paper_2603_11243_amd.pipeline import TwoPhaseDecoder
    wl = scaled_down(WORKLOADS[name], n_layers=layers, B=24 if layers and name.startswith("cfg3") else 4)
    cb, table = make_ctc_batch(wl), make_ctc_to_llm_map(wl)
    vi = make_verify_inputs(wl, cb.seconds, [np.zeros(0, np.int32)] * wl.B, device="cuda")
    ctx = Context(wl.model, make_model_weights(wl.model, wl.seed, device="cuda"))
    args = (ctx, wl, cb.logits.cuda(), cb.cu_frames, torch.from_numpy(table).cuda(), vi.speech_emb, vi.cu_speech, torch.from_numpy(vi.prompt_ids).cuda(), vi.cu_prompt)
    budget = 1500 if name.startswith("cfg3") else 200
    try:
        ctx.device_flags()
        resident = TwoPhaseDecoder(*args, budget=budget, n_steps=5).run(_tau_for(wl))
        assert resident["rejected"] > 0 and resident["verify_bins"] > 1
        for dtype in (ctx.act_dtype, torch.int8, torch.float8_e4m3fn):
            dec = TwoPhaseDecoder(*args, budget=budget, mode="paged", n_steps=5, pages_dtype=dtype, page_rows=16)
            for _ in range(2):                               # a second run on the same pages
                run = dec.run(_tau_for(wl))
                assert np.array_equal(run["accept_len"], resident["accept_len"]) and set(run["tokens"]) == set(resident["tokens"])
                for b, t in run["tokens"].items():
                    if dtype is ctx.act_dtype:
                        assert np.array_equal(t, resident["tokens"][b]), b
                    assert len(t) == 6 and t[0] == resident["tokens"][b][0] and (t >= 0).all() and (t < wl.model.vocab).all()
        assert ctx.device_flags() == 0
    finally:
        ctx.close()


@pytest.mark.parametrize("trees", [None, dict(tau=0.5, depth=4)])
def test_pages_with_trees_and_another_stream_current(trees):
    """The rows come back to slots with the room that trees take; the calls are queued while another stream than the context's is the current one."""
    from paper_2603_11243_amd.binding import Context
    from paper_2603_11243_amd.pipeline import TwoPhaseDecoder
    wl = WORKLOADS["cfg1_tiny_f32"]
    cb, table = make_ctc_batch(wl), make_ctc_to_llm_map(wl)
    vi = make_verify_inputs(wl, cb.seconds, [np.zeros(0, np.int32)] * wl.B, device="cuda")
    runs, side = [], torch.cuda.Stream()
    for mode, stream in (("resident", None), ("paged", side)):
        ctx = Context(wl.model, _weights(wl.model, 3), stream=stream)
        dec = TwoPhaseDecoder(ctx, wl, cb.logits.cuda(), cb.cu_frames, torch.from_numpy(table).cuda(), vi.speech_emb, vi.cu_speech,
                              torch.from_numpy(vi.prompt_ids).cuda(), vi.cu_prompt, budget=300, mode=mode, n_steps=9, trees=trees, pages_dtype=torch.float32, page_rows=32)
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(side):
                a = torch.randn(4096, 4096, device="cuda")
                for _ in range(100):                         # some tens of milliseconds
                    a = torch.matmul(a, a).clamp_(-1, 1)
        runs.append(dec.run(0.5))
        torch.cuda.synchronize()
        assert ctx.device_flags() == 0
        ctx.close()
    want, got = runs
    assert want["rejected"] > 0 and np.array_equal(got["accept_len"], want["accept_len"]) and set(got["tokens"]) == set(want["tokens"])
    assert all(np.array_equal(t, want["tokens"][b]) for b, t in got["tokens"].items())


def test_no_wait_inside_a_phase(monkeypatch):
    """Nothing between the bins of a phase waits for the stream: torch refuses copies that would while rows go to pages or come back."""
    from paper_2603_11243_amd.binding import Context
    from paper_2603_11243_amd.pipeline import TwoPhaseDecoder
    wl = scaled_down(WORKLOADS["cfg3_1b_ragged64"], n_layers=2, B=24)
    cb, table = make_ctc_batch(wl), make_ctc_to_llm_map(wl)
    vi = make_verify_inputs(wl, cb.seconds, [np.zeros(0, np.int32)] * wl.B, device="cuda")
    ctx = Context(wl.model, make_model_weights(wl.model, wl.seed, device="cuda"))
    dec = TwoPhaseDecoder(ctx, wl, cb.logits.cuda(), cb.cu_frames, torch.from_numpy(table).cuda(), vi.speech_emb, vi.cu_speech, torch.from_numpy(vi.prompt_ids).cuda(), vi.cu_prompt,
                          budget=1500, mode="paged", n_steps=5, page_rows=16)
    calls = []

    def watched(name):
        call = getattr(dec, name)

        def quiet(*args):
            torch.cuda.set_sync_debug_mode("error")
            try:
                call(*args)
            finally:
                torch.cuda.set_sync_debug_mode("default")
            calls.append(name)
        monkeypatch.setattr(dec, name, quiet)
    watched("_to_pages")
    watched("_from_pages")
    run = dec.run(_tau_for(wl))
    assert calls.count("_to_pages") == run["verify_bins"] > 1 and calls.count("_from_pages") == run["fallback_bins"] > 0
    ctx.close()
