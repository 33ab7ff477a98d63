"""Cases of the operators around a tree of drafted tokens: attention of its nodes over cached rows (with or without the weight that
every cached row collects), eviction of rows by that weight, and the accepted path of a tree.

`run` computes a case in its plain form, elementary torch operations in 32 bits, or, where `own` is true, by the framework's calls."""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
DEVICE = "cuda:0"


# ---- cases ---------------------------------------------------------------------------------------------------------------------
# attention: B utterances of ctx_lo .. ctx_hi cached rows and trees of nodes_lo .. nodes_hi nodes; `layout` is the order of the cache
# (slots: [slot][head][dim], the framework's own; heads: [head][slot][dim]); `lens` seeds lengths and trees.
def _attention(name, B, ctx, nodes, heads, dtype, layout="slots", shape="branches", mass=False, lens=1):
    c = {"op": "attention", "B": B, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "nodes_lo": nodes[0], "nodes_hi": nodes[1], "hq": heads[0], "hkv": heads[1],
         "hd": heads[2], "dtype": dtype, "layout": layout, "shape": shape, "mass": mass, "lens": lens}
    return dict(c, name=name) if name else c


def _evict(name, L, B, ctx, keep, heads, dtype, first, recent, lens=1):
    c = {"op": "evict", "L": L, "B": B, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "keep": keep, "hkv": heads[0], "hd": heads[1], "dtype": dtype,
         "first": first, "recent": recent, "lens": lens}
    return dict(c, name=name) if name else c


def _path(name, B, nodes, shape, tau, lens=1):
    c = {"op": "path", "B": B, "nodes_lo": nodes[0], "nodes_hi": nodes[1], "shape": shape, "tau": tau, "lens": lens}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one ten-second utterance of the 1B-class decoder, one new token: what a single decoding step costs
        _attention("one token", 1, (106, 106), (1, 1), (16, 8, 128), "f16"),
        # the utterances of a 64-utterance batch that failed the gate, a few candidates each
        _attention("small trees", 38, (60, 240), (4, 16), (16, 8, 128), "f16"),
        # the 3B-class decoder's batch with wide trees
        _attention("wide trees", 90, (100, 340), (32, 64), (24, 8, 128), "bf16", lens=3),
        # the small fp32 model
        _attention("fp32 trees", 4, (40, 70), (9, 20), (4, 4, 64), "f32"),
        # recordings of about an hour, cache ordered by head
        _attention("long recordings", 4, (20000, 40000), (16, 33), (16, 8, 128), "bf16", layout="heads", lens=5),
        # one context of a day's length: bytes alone
        _attention("one very long context", 1, (200001, 200001), (24, 24), (16, 8, 128), "f16"),
        # the small trees again, with the weight of every row
        _attention("small trees, weights", 38, (60, 240), (4, 16), (16, 8, 128), "f16", mass=True, lens=2),
        _attention("long recordings, weights", 2, (30000, 33000), (25, 31), (24, 8, 128), "bf16", mass=True, lens=7),
        # all layers of the 1B-class decoder, contexts cut to 128 rows
        _evict("evict, all layers", 24, 6, (200, 400), 128, (8, 128), "f16", 4, 32),
        # two layers of one long context
        _evict("evict, long context", 2, 1, (65537, 65537), 8191, (8, 128), "bf16", 16, 1000),
        _path("path of one tree", 1, (24, 24), "branches", 0.1),
        _path("paths of many trees", 256, (64, 1000), "branches", 0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    lens = rng.randrange(1, 1 << 20)
    shape = rng.choice(["branches", "chain", "wide"])
    kind = rng.choice(["attention", "attention", "weights", "evict", "path"])
    if kind in ("attention", "weights"):
        dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
        heads = (rng.choice([4, 8]),) * 2 + (64,) if dtype == "f32" else rng.choice([(16, 8, 128), (24, 8, 128), (8, 8, 128), (16, 4, 64), (8, 2, 128), (14, 2, 64)])
        B = _log_int(rng, 1, 96)
        most = 6000 if dtype == "f32" else 120000
        hi = _log_int(rng, 20, max(40, min(most, 160000 // B)))
        nodes = _log_int(rng, 1, min(96, max(2, 60000000 // (B * hi * heads[0]))))
        return _attention(None, B, (max(1, hi // rng.choice([1, 2, 4])), hi), (max(1, nodes // 2), nodes), heads, dtype, rng.choice(["slots", "heads"]), shape,
                          kind == "weights", lens)
    if kind == "evict":
        L = rng.choice([1, 2, 8, 24])
        B = _log_int(rng, 1, 16)
        hi = _log_int(rng, 100, 70000 // (L * B))
        keep = max(8, int(hi * rng.uniform(0.1, 0.6)))
        return _evict(None, L, B, (max(1, hi // 2), hi), keep, rng.choice([(8, 128), (4, 64), (2, 128)]), rng.choice(["f16", "bf16", "f32"]),
                      rng.randrange(0, keep // 4 + 1), rng.randrange(0, keep // 2 + 1), lens)
    hi = _log_int(rng, 1, 1000)
    return _path(None, _log_int(rng, 1, 256), (max(1, hi // 3), hi), shape, rng.choice([0.01, 0.1, 0.2, 0.5]), lens)


# ---- lengths and trees of a case -----------------------------------------------------------------------------------------------
def _tree(r, n, shape):
    if shape == "chain":
        return [i - 1 for i in range(n)]
    if shape == "wide":
        return [-1 if i < 2 else r.randrange(0, max(1, i // 4) + 1) for i in range(n)]
    return [-1 if i == 0 else i - 1 if r.random() < 0.6 else r.randrange(-1 if i < 3 else 0, i) for i in range(n)]


def _lengths(case):
    r = random.Random(case["lens"])
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["B"])] if "ctx_lo" in case else None
    trees = [_tree(r, r.randint(case["nodes_lo"], case["nodes_hi"]), case["shape"]) for _ in range(case["B"])] if "shape" in case else None
    return ctx, trees


def _starts(case, sizes):
    """Slots of the utterances: in some order, with a few free ones between them."""
    r = random.Random(case["lens"] + 1)
    order = list(range(len(sizes)))
    r.shuffle(order)
    start, at = [0] * len(sizes), 0
    for b in order:
        start[b] = at
        at += sizes[b] + r.randrange(4)
    return start, at


def _ancestors(trees):
    """[B, N, N] on the device: node j is i or an ancestor of i."""
    n = max(len(t) for t in trees)
    rows = [[t[i] if i < len(t) and t[i] >= 0 else n for t in trees] for i in range(n)]
    parent = torch.tensor(rows, device=DEVICE)
    seen = torch.zeros(len(trees), n + 1, n, dtype=torch.bool, device=DEVICE)
    every = torch.arange(len(trees), device=DEVICE)
    for i in range(n):
        seen[:, i] = seen[every, parent[i]]
        seen[:, i, i] = True
    return seen[:, :n]


def _index(values):
    return torch.tensor(values, dtype=torch.long, device=DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    ctx, trees = _lengths(case)
    s = {"case": case}
    if trees:
        s["parent"] = np.array([p for t in trees for p in t], dtype=np.int32)
        s["cu_nodes"] = np.cumsum([0] + [len(t) for t in trees]).astype(np.int32)
        n_max, N = max(len(t) for t in trees), len(s["parent"])
        s["ancestors"] = _ancestors(trees)
        s["node"] = (_index([b for b, t in enumerate(trees) for _ in t]), _index([i for t in trees for i in range(len(t))]))
        s["padded"] = _index([[min(i, len(t) - 1) for i in range(n_max)] for t in trees]) + _index(s["cu_nodes"][:-1].tolist())[:, None]
        s["lived"] = torch.arange(n_max, device=DEVICE) < _index([len(t) for t in trees])[:, None]
    if case["op"] == "path":
        # log-likelihoods of drafted tokens: most clearly above the threshold, some below it
        u = torch.rand(N, generator=g, device=DEVICE)
        s["logp"] = torch.where(torch.rand(N, generator=g, device=DEVICE) < 0.9, -0.3 * u, -2.0 - 6.0 * u)
        s["depth"] = s["ancestors"].sum(-1) - 1
        return s
    t, hkv, hd, B = TYPES[case["dtype"]], case["hkv"], case["hd"], case["B"]

    def rows_of(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device=DEVICE) * scale).to(t)

    if case["op"] == "attention":
        start, slots = _starts(case, [c + len(tr) for c, tr in zip(ctx, trees)])
        s["q"] = rows_of(N, case["hq"], hd, scale=2.0)

        def cache():
            return rows_of(slots, hkv, hd) if case["layout"] == "slots" else rows_of(hkv, slots, hd).transpose(0, 1)

        s["k"], s["v"] = cache(), cache()
        s["kv_start"], s["ctx_len"] = np.array(start, dtype=np.int32), np.array(ctx, dtype=np.int32)
        total = torch.tensor([c + len(tr) for c, tr in zip(ctx, trees)], device=DEVICE)[:, None]
        at, cl, first = torch.arange(int(total.max()), device=DEVICE), _index(ctx)[:, None], _index(start)[:, None]
        s["rows"] = first + torch.minimum(at, total - 1)
        # what a node sees: the context, its ancestors and itself
        in_tree = s["ancestors"].gather(2, (at - cl).clamp(0, n_max - 1)[:, None].expand(B, n_max, -1))
        s["seen"] = ((at < cl)[:, None] | (in_tree & (at >= cl)[:, None])) & (at < total)[:, None]
        if case["mass"]:
            s["mass"] = torch.rand(hkv, slots, generator=g, device=DEVICE) * (case["nodes_hi"] * case["hq"] / (hkv * case["ctx_hi"]))
            s["old"], s["valid"] = at < cl, at < total
        return s
    # eviction: weights as attention leaves them, most of them small, a few large
    start, slots = _starts(case, ctx)
    kept = [min(c, case["keep"]) for c in ctx]
    out_start, out_slots = np.cumsum([0] + kept)[:-1], sum(kept)
    L = case["L"]
    s["k"], s["v"] = rows_of(L, slots, hkv, hd), rows_of(L, slots, hkv, hd)
    s["mass"] = torch.randn(L, hkv, slots, generator=g, device=DEVICE).mul_(2.0).exp_()
    s["k_out"], s["v_out"] = (torch.empty(L, out_slots, hkv, hd, dtype=t, device=DEVICE) for _ in range(2))
    s["mass_out"] = torch.empty(L, hkv, out_slots, device=DEVICE)
    s["kv_start"], s["ctx_len"] = np.array(start, dtype=np.int32), np.array(ctx, dtype=np.int32)
    s["keep"], s["out_start"] = np.array(kept, dtype=np.int32), out_start.astype(np.int32)
    at, cl, first = torch.arange(max(ctx), device=DEVICE), _index(ctx)[:, None], _index(start)[:, None]
    s["rows"] = first + torch.minimum(at, cl - 1)
    s["always"] = (at < case["first"]) | (at >= cl - case["recent"])
    s["valid"] = at < cl
    s["kept"] = (_index([b for b, n in enumerate(kept) for _ in range(n)]), _index([i for n in kept for i in range(n)]))
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------------------
def _plain_attention(s):
    c = s["case"]
    hkv, hd, g = c["hkv"], c["hd"], c["hq"] // c["hkv"]
    B, n = s["padded"].shape
    k = s["k"][s["rows"]].float().permute(0, 2, 3, 1).contiguous()                       # [B, hkv, hd, rows]
    v = s["v"][s["rows"]].float().transpose(1, 2).contiguous()                           # [B, hkv, rows, hd]
    q = s["q"][s["padded"]].float().view(B, n, hkv, g, hd).permute(0, 2, 3, 1, 4).reshape(B, hkv, g * n, hd)
    score = torch.matmul(q, k).view(B, hkv, g, n, -1) * (1.0 / math.sqrt(hd))
    score = score.masked_fill(~s["seen"][:, None, None], float("-inf"))
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, hkv, g * n, -1), v).view(B, hkv, g, n, hd).permute(0, 3, 1, 2, 4).reshape(B, n, c["hq"], hd)
    out = o[s["node"]].to(s["q"].dtype)
    if not c["mass"]:
        return out
    weight = (p * s["lived"][:, None, None, :, None]).sum((2, 3))                        # [B, hkv, rows]
    before = s["mass"][:, s["rows"]].transpose(0, 1)                                     # [B, hkv, rows]
    after = torch.where(s["old"][:, None], before + weight, weight)
    s["mass"][:, s["rows"][s["valid"]]] = after.transpose(0, 1)[:, s["valid"]]
    return {"out": out, "mass": s["mass"]}


def _plain_evict(s):
    c = s["case"]
    w = s["mass"][:, :, s["rows"]]                                                       # [L, hkv, B, rows]
    w = torch.where(s["always"], math.inf, w)
    w = torch.where(s["valid"], w, -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices                  # equal ones: the lowest row first
    taken = torch.arange(order.shape[-1], device=DEVICE) < _index(s["keep"].tolist())[:, None]
    chosen = torch.zeros_like(w, dtype=torch.bool).scatter_(-1, order, taken.expand_as(order))
    rows = torch.sort(chosen.to(torch.int8), dim=-1, descending=True, stable=True).indices[:, :, s["kept"][0], s["kept"][1]]    # [L, hkv, kept]
    slot = s["rows"][s["kept"][0], rows]
    per_head = slot.transpose(1, 2)[..., None].expand(-1, -1, -1, c["hd"])
    torch.gather(s["k"], 1, per_head, out=s["k_out"])
    torch.gather(s["v"], 1, per_head, out=s["v_out"])
    torch.gather(s["mass"], 2, slot, out=s["mass_out"])
    return {"k": s["k_out"], "v": s["v_out"], "mass": s["mass_out"], "rows": rows.to(torch.int32)}


def _plain_path(s):
    B, n = s["padded"].shape
    fails = ~(s["logp"][s["padded"]] > float(np.float32(math.log(s["case"]["tau"])))) & s["lived"]
    good = ~(s["ancestors"] & fails[:, None]).any(-1) & s["lived"]
    depth = torch.where(good, s["depth"], -1)
    deepest = depth.amax(1)
    number = torch.arange(n, device=DEVICE)
    best = torch.where(depth == deepest[:, None], number, n).amin(1)
    accepted = deepest + 1
    on_path = s["ancestors"].gather(1, best.clamp(max=n - 1)[:, None, None].expand(B, 1, n))[:, 0] & (accepted > 0)[:, None] & s["lived"]
    path = torch.full((B, n + 1), -1, dtype=torch.long, device=DEVICE)
    path.scatter_(1, torch.where(on_path, s["depth"], n), torch.where(on_path, number, -1).expand(B, n))
    return {"accept_len": accepted.to(torch.int32), "accept_node": torch.where(accepted > 0, best, -1).to(torch.int32),
            "path": path[s["node"]].to(torch.int32)}


# ---- the framework's calls -----------------------------------------------------------------------------------------------------
_contexts = {}


def _context(s):
    """One context for the whole program, its workspace large enough for this state."""
    if "ctx" not in s:
        from paper_2603_11243_amd.binding import Context
        c = s["case"]
        ctx = _contexts.setdefault(DEVICE, None) or Context(device=DEVICE)
        _contexts[DEVICE] = ctx
        if c["op"] == "attention":
            ctx.reserve(tree_nodes=len(s["parent"]), tree_utts=c["B"], tree_heads=(c["hq"], c["hkv"], c["hd"]))
        elif c["op"] == "evict":
            ctx.reserve(evict_rows=int(s["keep"].sum()), evict_utts=c["B"], evict_heads=(c["L"], c["hkv"]))
        else:
            ctx.reserve(tree_nodes=len(s["parent"]), tree_utts=c["B"])
        s["ctx"] = ctx
    return s["ctx"]


def run(s):
    c = s["case"]
    if not own:
        return {"attention": _plain_attention, "evict": _plain_evict, "path": _plain_path}[c["op"]](s)
    ctx = _context(s)
    if c["op"] == "attention":
        out = ctx.tree_attention(s["q"], s["k"], s["v"], s["kv_start"], s["ctx_len"], s["cu_nodes"], s["parent"], mass=s.get("mass"))
        return {"out": out, "mass": s["mass"]} if c["mass"] else out
    if c["op"] == "evict":
        rows = ctx.kv_evict(s["k"], s["v"], s["mass"], s["kv_start"], s["ctx_len"], s["keep"], c["first"], c["recent"], s["k_out"], s["v_out"],
                            s["out_start"], mass_out=s["mass_out"], want_rows=True)
        return {"k": s["k_out"], "v": s["v_out"], "mass": s["mass_out"], "rows": rows}
    return ctx.tree_path(s["logp"], s["cu_nodes"], s["parent"], c["tau"])


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------------
def work(case):
    ctx, trees = _lengths(case)
    es = {"f16": 2, "bf16": 2, "f32": 4}.get(case.get("dtype"), 0)
    if case["op"] == "path":
        n = sum(len(t) for t in trees)
        return {"bytes": 4 * n + 4 * n + 8 * case["B"], "flops": 2 * n}
    if case["op"] == "evict":
        kept = sum(min(c, case["keep"]) for c in ctx)
        heads = case["L"] * case["hkv"]
        return {"bytes": heads * (4 * sum(ctx) + 8 * kept + 4 * kept * case["hd"] * es), "flops": heads * sum(ctx)}
    nodes, rows = sum(len(t) for t in trees), sum(ctx) + sum(len(t) for t in trees)
    pairs = 0
    for c, t in zip(ctx, trees):
        depth = []
        for p in t:
            depth.append(1 if p < 0 else depth[p] + 1)
        pairs += c * len(t) + sum(depth)
    w = {"bytes": 2 * rows * case["hkv"] * case["hd"] * es + 2 * nodes * case["hq"] * case["hd"] * es, "flops": 4 * pairs * case["hq"] * case["hd"]}
    if case["mass"]:
        w["bytes"] += 4 * case["hkv"] * (2 * sum(ctx) + nodes)
    return w


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    ctx, trees = _lengths(case)
    if case["op"] == "path":
        logp, lengths, best, path = s["logp"].double().cpu().tolist(), [], [], []
        for b, t in enumerate(trees):
            depth = []                                       # of nodes that stand, 0 for the others
            for i, p in enumerate(t):
                above = 1 if p < 0 else depth[p] + 1 if depth[p] else 0
                depth.append(above if logp[int(s["cu_nodes"][b]) + i] > float(np.float32(math.log(case["tau"]))) else 0)
            n = max(depth)
            at = depth.index(n) if n else -1
            lengths.append(n)
            best.append(at)
            up = []
            while at >= 0:
                up.append(at)
                at = t[at]
            path += up[::-1] + [-1] * (len(t) - n)
        return {"accept_len": np.array(lengths, np.int32), "accept_node": np.array(best, np.int32), "path": np.array(path, np.int32)}
    if case["op"] == "evict":
        L, hkv = case["L"], case["hkv"]
        mass, chosen = s["mass"].cpu().numpy(), []
        for b, n in enumerate(ctx):
            m = mass[:, :, s["kv_start"][b]:s["kv_start"][b] + n].astype(np.float64)
            m[:, :, :case["first"]] = np.inf
            m[:, :, max(0, n - case["recent"]):] = np.inf
            chosen.append(np.sort(np.argsort(-m, axis=-1, kind="stable")[:, :, :min(n, case["keep"])], axis=-1))
        rows = np.concatenate(chosen, -1)
        slots = torch.from_numpy(np.concatenate([x + int(a) for x, a in zip(chosen, s["kv_start"])], -1)).to(DEVICE)
        layer, head = torch.arange(L, device=DEVICE)[:, None, None], torch.arange(hkv, device=DEVICE)[None, :, None]
        return {"k": s["k"][layer, slots, head].transpose(1, 2), "v": s["v"][layer, slots, head].transpose(1, 2),
                "mass": s["mass"][layer, head, slots], "rows": rows.astype(np.int32)}
    g = case["hq"] // case["hkv"]
    out = torch.zeros(len(s["parent"]), case["hq"], case["hd"], dtype=torch.float64, device=DEVICE)
    mass = s["mass"].double() if case["mass"] else None
    for b, (n, t) in enumerate(zip(ctx, trees)):
        a, z, node = int(s["kv_start"][b]), int(s["kv_start"][b]) + n + len(t), int(s["cu_nodes"][b])
        sees = np.zeros((len(t), n + len(t)), dtype=bool)
        sees[:, :n] = True
        for i in range(len(t)):
            at = i
            while at >= 0:
                sees[i, n + at] = True
                at = t[at]
        hidden = torch.from_numpy(~sees).to(DEVICE)
        for h in range(case["hkv"]):
            k, v = s["k"][a:z, h].double(), s["v"][a:z, h].double()
            total = torch.zeros(z - a, dtype=torch.float64, device=DEVICE)
            for j in range(h * g, (h + 1) * g):
                w = torch.softmax((s["q"][node:node + len(t), j].double() @ k.T / math.sqrt(case["hd"])).masked_fill(hidden, -math.inf), -1)
                out[node:node + len(t), j] = w @ v
                total += w.sum(0)
            if mass is not None:
                mass[h, a:a + n] += total[:n]
                mass[h, a + n:z] = total[n:]
    return {"out": out, "mass": mass} if case["mass"] else out
