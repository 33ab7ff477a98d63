"""TreeFallback beside ar_fallback: 16-bit models, utterance by utterance; utterances alone and in a batch."""
import numpy as np
import pytest
import torch

from tests import test_gpu_verify_tree as rounds
from tests.parity import TOL_LOGP
from tests.test_gpu_tree_attention import Call, _batch, _context
from trees import cu, flat

pytestmark = pytest.mark.gpu

PEAK = 12.0


def _peaked(m, seed):
    w = rounds.make_model_weights(m, seed, device="cuda")
    w["lm_head"] = (w["lm_head"].float() * PEAK).to(w["lm_head"].dtype)
    return w


# Logits are PEAK times those of the other tests, and so are their errors: tol.  ar_fallback's choice is at most 2 tol below the other in exact numbers, the
# trees' choice at most 2 tol below ar_fallback's, and the pass that compares them is off by tol for each.
@pytest.mark.parametrize("name", ["1b_half", "1b_bfloat16"])
@pytest.mark.parametrize("depth", [2, 5])
def test_16_bit_continuations_part_at_near_ties_only(name, depth, monkeypatch):
    from paper_2603_11243_amd.pipeline import TreeFallback
    monkeypatch.setattr(rounds, "_weights", _peaked)
    n_steps, prompts = 20, [30, 45, 12, 70, 5, 22]
    B = len(prompts)
    ctx, m, w, start, r = rounds._prefilled(name, prompts, n_steps + 30)
    tol = PEAK * TOL_LOGP[m.dtype] * (8 if ctx.act_dtype == torch.bfloat16 else 1)
    ctx.reserve(ar_utts=B, ar_steps=n_steps)
    first = np.array([3, 5, 7, 11, 13, 17], dtype=np.int32)
    want = ctx.ar_fallback(start, prompts, torch.from_numpy(first).cuda(), n_steps).cpu().numpy()
    drafts = []
    for b in range(B):                                       # the rejected token, then that continuation with a token replaced, left out or put in
        d = [1] + want[:, b].tolist()
        if b % 4 == 1:
            d[4] = 2
        if b % 4 == 2:
            del d[3]
        if b % 4 == 3:
            d.insert(5, 9)
        drafts.append(np.array(d, dtype=np.int32))
    passes, inner = [], ctx.verify_tree
    monkeypatch.setattr(ctx, "verify_tree", lambda *a, **k: passes.append(1) or inner(*a, **k))
    got = TreeFallback(ctx, B, tau=0.5, depth=depth).run(start, prompts, first, drafts, n_steps)
    monkeypatch.undo()
    same = [int(np.argmin(np.append(g[1:] == want[:, b], False))) for b, g in enumerate(got)]
    print(f"{name}: {len(passes)} passes for {n_steps} tokens, equal up to {same}")
    assert len(passes) < n_steps
    trees, ids = [], []
    for b, k in enumerate(same):
        assert len(got[b]) == n_steps + 1 and got[b][0] == first[b]
        k = min(k, n_steps - 1)
        trees.append([i - 1 for i in range(k + 1)] + [k, k])
        ids += got[b][:k + 1].tolist() + [int(want[k, b]), int(got[b][k + 1])]
    ids = torch.tensor(ids, dtype=torch.int32, device="cuda")
    h = ctx.verify_tree(ids, cu(trees), flat(trees), start, prompts)
    logp = ctx.accept_tree(h, ids, cu(trees), flat(trees), 0.5)["node_logp"].cpu().numpy()
    for b, end in enumerate(cu(trees)[1:]):
        gap = abs(logp[end - 1] - logp[end - 2])
        print(f"utterance {b}: {gap:.3f} between the candidates at {same[b]}")
        assert gap <= 6 * tol, (b, same[b])
    ctx.close()


@pytest.mark.parametrize("dtype, heads", [("f16", (16, 8, 128)), ("bf16", (4, 2, 64)), ("f32", (4, 2, 36))])
def test_utterances_alone_and_together(dtype, heads):
    """The same bits where tiles and pieces are the same (trees of a size, contexts that are not cut), the error bound where the batch changes them."""
    ctx_len, nodes = [50, 70, 90, 0, 333], [6, 6, 5, 6, 4]
    trees = _batch(71, None, nodes)

    def one(c, b):
        alone = Call.__new__(Call)
        alone.__dict__.update(c.__dict__)
        at = slice(int(cu(c.trees)[b]), int(cu(c.trees)[b + 1]))
        alone.trees, alone.ctx_len, alone.kv_start = [c.trees[b]], c.ctx_len[b:b + 1], c.kv_start[b:b + 1]
        alone.q, alone.lse = c.q[at], c.lse[at].clone()
        return alone, at
    for mixed in (False, True):
        c = Call(dtype, heads, ctx_len + [9000] * mixed, trees + [[-1] * 70] * mixed, seed=72)
        c.check(_context(200, 6, heads))
        whole, mass = c.run().clone(), c.mass_out.clone()
        for b in range(5):
            alone, at = one(c, b)
            got = alone.run()
            rows = slice(int(c.kv_start[b]), int(c.kv_start[b]) + ctx_len[b] + nodes[b])
            if mixed:
                used = torch.zeros_like(c.used)
                used[rows] = True
                alone.used = used
                alone.check()
            else:
                assert torch.equal(got, whole[at]) and torch.equal(alone.mass_out[:, rows], mass[:, rows])
