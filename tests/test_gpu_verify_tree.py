"""verify_tree and accept_tree against a decoder pass in 64 bits over the very rows of the K/V cache, rounds after one another, and the tree
fallback against ar_fallback."""
from dataclasses import replace

import numpy as np
import pytest
import torch

from oracle import ssd_oracle as O
from tests.parity import TOL_LOGP
from trees import accepted, cu, flat, path_to, sees, tree
from workloads import WORKLOADS, make_model_weights
from workloads.configs import LLM_1B, LLM_3B, TINY, ModelCfg

pytestmark = pytest.mark.gpu

MODELS = {"tiny": (TINY, "f16"), "f32_group": (ModelCfg(n_layers=2, d_model=96, n_q_heads=4, n_kv_heads=2, head_dim=36, d_ff=128, vocab=512, dtype="f32"), "f16"),
          "1b_half": (replace(LLM_1B, n_layers=2), "f16"), "1b_bfloat16": (replace(LLM_1B, n_layers=2), "bf16"), "3b_half": (replace(LLM_3B, n_layers=1), "f16")}


def _weights(m, seed):
    """Peaked distributions for the fp32 models, so that tokens are far from ties."""
    w = make_model_weights(m, seed, device="cuda")
    if m.dtype == "f32":
        g = torch.Generator(device="cuda").manual_seed(seed)
        for L in w["layers"]:
            for k in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down"):
                L[k] = torch.randn(L[k].shape, generator=g, device="cuda") * 0.08
        w["lm_head"] = torch.randn(w["lm_head"].shape, generator=g, device="cuda") * 0.3
        w["embed"] = torch.randn(w["embed"].shape, generator=g, device="cuda") * 0.5
    return w


def _nodes_exact(w, m, k, v, ids, parent, pos0):
    """Nodes of one tree over cached rows k, v [layers, n, K/V heads, head_dim]: (final-normed rows, per layer the weight of every row
    [layers, K/V heads, n + nodes]), by the decoder layer of the oracle with the node's rows in place of the causal ones."""
    n, N, hq, hkv, hd = k.shape[1], len(parent), m.n_q_heads, m.n_kv_heads, m.head_dim
    pos = np.array([pos0 + len(path_to(parent, i)) - 1 for i in range(N)])
    seen = np.concatenate([np.ones((N, n), bool), sees(parent)], 1)
    x = O._f64(w["embed"][torch.from_numpy(ids).long().to(w["embed"].device)])
    weights = np.zeros((m.n_layers, hkv, n + N))
    for l, L in enumerate(w["layers"]):
        L = {name: O._f64(t) for name, t in L.items()}
        a = O.rmsnorm(x, L["norm_attn"], m.rms_eps)
        q = O.rope((a @ L["wq"].T).reshape(N, hq, hd), pos, m.rope_theta)
        kk = np.concatenate([k[l], O.rope((a @ L["wk"].T).reshape(N, hkv, hd), pos, m.rope_theta)])
        vv = np.concatenate([v[l], (a @ L["wv"].T).reshape(N, hkv, hd)])
        o = np.zeros((N, hq, hd))
        for h in range(hq):
            g = h * hkv // hq
            s = np.where(seen, q[:, h] @ kk[:, g].T / np.sqrt(hd), -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[:, h] = p @ vv[:, g]
            weights[l, g] += p.sum(0)
        x = x + o.reshape(N, -1) @ L["wo"].T
        b = O.rmsnorm(x, L["norm_mlp"], m.rms_eps)
        x = x + (O.silu(b @ L["w_gate"].T) * (b @ L["w_up"].T)) @ L["w_down"].T
    return O.rmsnorm(x, O._f64(w["norm_final"]), m.rms_eps), weights


def _prefilled(name, prompts, room, slots_more=0, seed=5):
    """A context whose cache holds the rows of `prompts` prompt tokens an utterance, and room slots behind them."""
    from paper_2603_11243_amd.binding import Context
    m, operand = MODELS[name]
    w = _weights(m, seed)
    ctx = Context(m, w, operand=operand)
    B = len(prompts)
    start = (np.cumsum(np.array(prompts) + room) - prompts - room).astype(np.int32)
    slots = int(sum(prompts) + B * room + slots_more)
    ctx.set_kv_cache(slots)
    ctx._kv.zero_()
    ctx.reserve(max_tokens=sum(prompts) + B, max_verify_rows=B, max_utts=B, tree_nodes=B * room, tree_utts=B)
    r = np.random.default_rng(seed)
    ids = torch.from_numpy(r.integers(0, m.vocab, size=sum(prompts)).astype(np.int32)).cuda()
    none = np.zeros(B + 1, np.int32)
    speech = torch.zeros(0, m.d_model, dtype=ctx.dtype, device="cuda")
    ctx.verify_forward(speech, none, ids, np.concatenate([[0], np.cumsum(prompts)]), ids[:0], none, kv_start=start)
    torch.cuda.synchronize()
    return ctx, m, w, start, r


def _rows(ctx, start, n):
    k, v = ctx.kv_tensors()
    return k[:, start:start + n].double().cpu().numpy(), v[:, start:start + n].double().cpu().numpy()


# Likelihoods within the tolerance of the other calls' tests, which is that of IEEE half operands: half a step is 2^-11 there and 2^-8 with bfloat16
# operands, every rounding of the pass is one to the operand type, so that each error is eight times as large; weights: sums of probabilities whose scores are off by about a rounding of q and k to the
# operand type each (eps / 2 relative each, scores below 16 here: 2 * 16 * eps / 2) and what the layers before left, another 4 eps of them; fp32: 2^-14.
@pytest.mark.parametrize("name", list(MODELS))
@pytest.mark.parametrize("prompts, nodes", [([17], [1]), ([40, 3, 100, 64], [9, 1, 20, 16]), ([30, 31, 90, 2, 33], [40, 33, 50, 1, 45])])
def test_rounds(name, prompts, nodes):
    ctx, m, w, start, r = _prefilled(name, prompts, max(nodes) * 2)
    tol, w_lm = TOL_LOGP[m.dtype] * (8 if ctx.act_dtype == torch.bfloat16 else 1), O._f64(w["lm_head"])
    eps = torch.finfo(ctx.act_dtype).eps
    w_tol = 2.0 ** -14 if m.dtype == "f32" else 20 * eps
    length, B = np.array(prompts, dtype=np.int32), len(prompts)
    k, _ = ctx.kv_tensors()
    mass = torch.zeros(k.shape[0], k.shape[2], k.shape[1], device="cuda")
    tau = 0.5 / m.vocab if m.dtype == "bf16" else 1e-3
    for turn in range(2):
        trees = [tree(r, n, ("random", "star", "random", "chain")[b % 4]) for b, n in enumerate(nodes)]
        N, at = sum(nodes), cu(trees)
        ids = r.integers(0, m.vocab, size=N).astype(np.int32)
        before = [_rows(ctx, start[b], length[b]) for b in range(B)]
        old = mass.double().cpu().numpy()
        t_ids = torch.from_numpy(ids).cuda()
        h = ctx.verify_tree(t_ids, at, flat(trees), start, length, kv_mass=mass)
        torch.cuda.synchronize()
        got_m, new_rows = mass.double().cpu().numpy(), [_rows(ctx, start[b] + length[b], nodes[b]) for b in range(B)]
        acc = ctx.accept_tree(h, t_ids, at, flat(trees), tau, kv_start=start, ctx_len=length, kv_mass=mass)
        torch.cuda.synchronize()
        got = {key: x.cpu().numpy() for key, x in acc.items()}
        for b, t in enumerate(trees):
            mine = slice(at[b], at[b + 1])
            hid, weights = _nodes_exact(w, m, *before[b], ids[mine], t, int(length[b]))
            logits = hid @ w_lm.T
            lse = np.log(np.exp(logits - logits.max(1, keepdims=True)).sum(1)) + logits.max(1)
            logp, greedy = got["node_logp"][mine], got["greedy_tok"][mine]
            for i, p in enumerate(t):
                if p < 0:
                    assert logp[i] == 0
                else:
                    assert abs(logp[i] - (logits[p, ids[mine][i]] - lse[p])) <= tol
                assert logits[i].max() - logits[i, greedy[i]] <= tol
            want = accepted(t, logp, tau, roots_given=True)
            assert got["accept_len"][b] == len(want) and got["accept_node"][b] == (want[-1] if want else -1)
            assert got["path"][mine].tolist() == want + [-1] * (len(t) - len(want))
            rows = slice(start[b], start[b] + length[b] + nodes[b])
            weights[:, :, :length[b]] += old[:, :, start[b]:start[b] + length[b]]
            assert (abs(got_m[:, :, rows] - weights) <= w_tol * weights + 1e-6).all()
            # the accepted rows, moved behind the context with their weights, as they were
            for x, y in zip(_rows(ctx, start[b] + length[b], len(want)), new_rows[b]):
                assert np.array_equal(x, y[:, want])
            for x, y in zip(_rows(ctx, start[b], length[b]), before[b]):
                assert np.array_equal(x, y)
            s0 = start[b] + length[b]
            assert np.array_equal(mass[:, :, s0:s0 + len(want)].double().cpu().numpy(), got_m[:, :, s0 + np.array(want, dtype=int)])
        length = length + got["accept_len"]
    ctx.close()


@pytest.mark.parametrize("name", ["tiny", "1b_half"])
def test_a_chain_is_what_verify_forward_makes_of_a_draft(name):
    ctx, m, w, start, r = _prefilled(name, [25, 60], 40)
    U = [12, 30]
    ids = torch.from_numpy(r.integers(0, m.vocab, size=sum(U)).astype(np.int32)).cuda()
    trees = [[i - 1 for i in range(n)] for n in U]
    h = ctx.verify_tree(ids, cu(trees), flat(trees), start, [25, 60])
    acc = ctx.accept_tree(h, ids, cu(trees), flat(trees), 0.0)
    assert acc["accept_len"].tolist() == U
    from paper_2603_11243_amd.binding import Context
    other = Context(m, w)
    other.reserve(max_tokens=200, max_verify_rows=60, max_utts=2)
    prompt = torch.from_numpy(np.random.default_rng(5).integers(0, m.vocab, size=85).astype(np.int32)).cuda()
    none = np.zeros(3, np.int32)
    hv = other.verify_forward(torch.zeros(0, m.d_model, dtype=ctx.dtype, device="cuda"), none, prompt, [0, 25, 85], ids, cu(trees))
    want = other.accept_prefix(hv, ids, cu(trees), 0.0, want_greedy=True)
    torch.cuda.synchronize()
    a, b = acc["node_logp"].cpu().numpy(), want["draft_logp"].cpu().numpy()
    for lo, n in zip(cu(trees), U):
        assert abs(a[lo + 1:lo + n] - b[lo + 1:lo + n]).max() <= 2 * TOL_LOGP[m.dtype]


def test_positions_after_eviction():
    """Contexts cut to some of their rows: the nodes go on at the position the whole one had."""
    ctx, m, w, start, r = _prefilled("tiny", [50, 80], 30)
    k, v = ctx.kv_tensors()
    mass = torch.rand(k.shape[0], k.shape[2], k.shape[1], device="cuda")
    slots = 150
    buf = torch.zeros(ctx.kv_cache_bytes(slots), dtype=torch.uint8, device="cuda")
    k2, v2 = ctx.kv_tensors(buf, slots)
    ctx.reserve(evict_rows=80, evict_utts=2, evict_heads=(m.n_layers, m.n_kv_heads))
    rows = ctx.kv_evict(k, v, mass, start, [50, 80], [20, 30], 2, 5, k2, v2, [70, 3], want_rows=True).cpu()
    kept = k2[1, 70:90, 2].clone()
    assert torch.equal(kept, k[1, int(start[0]) + rows[1, 2, :20].long(), 2])
    ctx.attach_kv_cache(buf, slots)
    trees, ids = [[-1, 0, 0, 1], [-1, 0]], np.arange(7, 13, dtype=np.int32)
    before = [_rows(ctx, 70, 20), _rows(ctx, 3, 30)]
    h = ctx.verify_tree(torch.from_numpy(ids).cuda(), cu(trees), flat(trees), [70, 3], [20, 30], pos0=[50, 80])
    torch.cuda.synchronize()
    h = h.double().cpu().numpy()
    for b, at, n0 in ((0, slice(0, 4), 50), (1, slice(4, 6), 80)):
        want, _ = _nodes_exact(w, m, *before[b], ids[at], trees[b], n0)
        assert abs(h[at] - want).max() <= 1e-4 * abs(want).max()


def test_refusals():
    from paper_2603_11243_amd.binding import SsdError
    ctx, m, w, start, r = _prefilled("tiny", [20, 20], 10)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    args = lambda **k: dict(dict(node_ids=ids, cu_nodes=[0, 2, 4], parent=[-1, 0, -1, 0], kv_start=start, ctx_len=[20, 20]), **k)
    h = ctx.verify_tree(**args())
    for bad in (dict(parent=[-1, 1, -1, 0]), dict(kv_start=[0, 21]), dict(ctx_len=[20, 49]), dict(pos0=[-1, 20]), dict(ctx_len=[-1, 20])):
        with pytest.raises(SsdError) as e:
            ctx.verify_tree(**args(**bad))
        assert e.value.code == -1
    with pytest.raises(SsdError) as e:
        ctx.verify_tree(**args(pos0=[1023, 20]))
    assert e.value.code == -2
    with pytest.raises(SsdError):
        ctx.accept_tree(h, ids, [0, 2, 4], [-1, 0, -1, 0], float("nan"))
    with pytest.raises(ValueError):
        ctx.verify_tree(**args(kv_mass=torch.zeros(5, device="cuda")))
    with pytest.raises(ValueError):
        ctx.verify_tree(**args(node_ids=ids.long()))
    assert ctx.verify_tree(ids[:0], [0, 0, 0], [], start, [20, 20]).shape == (0, m.d_model)
    ctx.set_workspace(None)
    with pytest.raises(SsdError) as e:
        ctx.verify_tree(**args())
    assert e.value.code == -3


@pytest.mark.parametrize("name", ["tiny", "1b_half"])
def test_tree_fallback_is_the_greedy_continuation(name):
    """tau 0.5: what the trees accept is what ar_fallback would choose.  The drafts are that continuation with a token replaced, left out or put in."""
    from paper_2603_11243_amd.pipeline import TreeFallback
    n_steps, prompts = 14, [30, 45, 12, 70]
    ctx, m, w, start, r = _prefilled(name, prompts, n_steps + 30)
    ctx.reserve(ar_utts=4, ar_steps=n_steps)
    first = np.array([3, 5, 7, 11], dtype=np.int32)
    want = ctx.ar_fallback(start, prompts, torch.from_numpy(first).cuda(), n_steps).cpu().numpy()
    drafts = []
    for b in range(4):
        d = [1] + want[:, b].tolist()                        # the rejected token, then the continuation
        if b == 1:
            d[4] = 2
        if b == 2:
            del d[3]
        if b == 3:
            d.insert(5, 9)
        drafts.append(np.array(d, dtype=np.int32))
    passes = []
    fallback = TreeFallback(ctx, 4, tau=0.5, depth=4)
    inner = ctx.verify_tree
    ctx.verify_tree = lambda *a, **k: passes.append(1) or inner(*a, **k)
    got = fallback.run(start, prompts, first, drafts, n_steps)
    same = [int(np.argmin(np.append(g[1:] == want[:, b], False))) for b, g in enumerate(got)]
    assert all(len(g) == n_steps + 1 and g[0] == first[b] for b, g in enumerate(got))
    print(f"{name}: {len(passes)} passes for {n_steps} tokens, equal up to {same}")
    if name == "tiny":                                       # (two sums of 16 bits may part at a near-tie)
        assert same == [n_steps] * 4
    assert sum(same) >= n_steps


def test_tree_fallback_with_short_contexts():
    """Contexts cut again and again: runs to the end, and the attached cache is the caller's again."""
    from paper_2603_11243_amd.pipeline import TreeFallback
    n_steps, prompts = 40, [60, 90]
    ctx, m, w, start, r = _prefilled("tiny", prompts, n_steps + 30)
    kv, rows = ctx._kv, _rows(ctx, start[0], 60)
    fallback = TreeFallback(ctx, 2, tau=0.0, depth=5, most_rows=64, keep_rows=40, n_first=2, n_recent=8)
    drafts = [r.integers(0, m.vocab, size=30).astype(np.int32) for _ in prompts]
    got = fallback.run(start, prompts, [1, 2], drafts, n_steps)
    assert [len(g) for g in got] == [n_steps + 1] * 2 and all((0 <= g).all() and (g < m.vocab).all() for g in got)
    assert ctx._kv is kv and all(np.array_equal(a, b) for a, b in zip(rows, _rows(ctx, start[0], 60)))
    assert got[0][1:5].tolist() == drafts[0][1:5].tolist()   # tau 0 takes the draft
    again = fallback.run(start, prompts, [1, 2], drafts, n_steps)
    assert all(np.array_equal(a, b) for a, b in zip(got, again))
