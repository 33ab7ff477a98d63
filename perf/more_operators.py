"""Cases of the operators around K/V rows in pages: writing rows into pages (as they are, or quantised to 8 bits with a scale per row and
head), reading them back, and attention of the newest tokens over the pages of their utterances.

`run` computes a case in its plain form, elementary torch operations in 32 bits (64 where a value lies next to the border between two codes),
or, where `own` is true, by the framework's calls."""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
SIZE = {"f16": 2, "bf16": 2, "f32": 4, "e4m3": 1, "i8": 1}
DEVICE = "cuda:0"


# ---- cases ---------------------------------------------------------------------------------------------------------------------
# attention: B utterances of ctx_lo .. ctx_hi rows, the newest `new` tokens of each attend; heads (query heads, K/V heads, head_dim).
def _attention(name, B, ctx, heads, q, pages, page_rows, new=1, lens=1):
    c = {"op": "attention", "B": B, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "hq": heads[0], "hkv": heads[1], "hd": heads[2], "dtype": q, "pages": pages,
         "page_rows": page_rows, "new": new, "lens": lens}
    return dict(c, name=name) if name else c


# write and read: L layers, B utterances whose last rows_lo .. rows_hi rows (of up to `before` more) go to or come from a cache of type dtype.
def _move(name, op, L, B, rows, before, heads, dtype, pages, page_rows, lens=1):
    c = {"op": op, "L": L, "B": B, "rows_lo": rows[0], "rows_hi": rows[1], "before": before, "hkv": heads[0], "hd": heads[1], "dtype": dtype, "pages": pages,
         "page_rows": page_rows, "lens": lens}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one ten-second utterance of the 1B-class decoder, one new token: what a single decoding step costs
        _attention("one token", 1, (106, 106), (16, 8, 128), "f16", "f16", 16),
        # the utterances of a 64-utterance batch that failed the gate, one decoding step
        _attention("38 utterances, e4m3", 38, (60, 240), (16, 8, 128), "f16", "e4m3", 16, lens=2),
        # the 3B-class decoder's batch, four drafted tokens behind each context
        _attention("90 utterances, i8, four tokens", 90, (100, 340), (24, 8, 128), "bf16", "i8", 32, new=4, lens=3),
        # the small fp32 model
        _attention("fp32", 4, (40, 70), (4, 4, 64), "f32", "f32", 16),
        # recordings of about an hour, 8-bit pages
        _attention("long recordings, e4m3", 4, (20000, 40000), (16, 8, 128), "bf16", "e4m3", 64, lens=5),
        # many contexts of some minutes, drafted tokens behind them: more query rows than one tile holds
        _attention("16 contexts, i8, nine tokens", 16, (1000, 9000), (24, 8, 128), "bf16", "i8", 64, new=9, lens=6),
        # one context of a day's length in 16 bits: bytes alone
        _attention("one very long context", 1, (200001, 200001), (16, 8, 128), "bf16", "bf16", 128),
        # the new rows of one layer in a decoding step
        _move("append one row each, e4m3", "write", 1, 64, (1, 1), 300, (8, 128), "f16", "e4m3", 16, lens=2),
        # all layers of the 1B-class decoder: rows of rejected utterances parked in 8 bits
        _move("park, all layers, i8", "write", 24, 6, (200, 400), 0, (8, 128), "f16", "i8", 64, lens=3),
        _move("park, long, e4m3", "write", 2, 1, (65537, 65537), 100, (8, 128), "bf16", "e4m3", 128),
        # and read back for the fallback
        _move("read back, few rows, i8", "read", 1, 4, (40, 70), 0, (4, 64), "f32", "i8", 16, lens=4),
        _move("read back, all layers, e4m3", "read", 24, 6, (200, 400), 0, (8, 128), "f16", "e4m3", 64, lens=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    lens = rng.randrange(1, 1 << 20)
    page_rows = rng.choice([16, 32, 64, 128])
    kind = rng.choice(["attention", "attention", "attention", "write", "read"])
    if kind == "attention":
        q = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
        pages = rng.choice([q, "e4m3", "i8"])
        heads = rng.choice([(16, 8, 128), (24, 8, 128), (8, 8, 128), (16, 4, 64), (8, 2, 128), (14, 2, 64), (4, 4, 64), (32, 1, 128)])
        B = _log_int(rng, 1, 96)
        hi = _log_int(rng, 20, max(40, min(120000, (90000 if pages == "f32" else 160000) // B)))
        new = rng.choice([1, 1, 1, 2, 4, 7])
        return _attention(None, B, (max(1, hi // rng.choice([1, 2, 4])), hi), heads, q, pages, page_rows, new, lens)
    L, B = rng.choice([1, 2, 8, 24]), _log_int(rng, 1, 48)
    dtype = rng.choice(["f16", "bf16", "f32"])
    pages = rng.choice([dtype, "e4m3", "i8", "e4m3", "i8"])
    hi = _log_int(rng, 1, max(2, 48000 // (L * B)))
    return _move(None, kind, L, B, (max(1, hi // 2), hi), rng.choice([0, 30, 500]) if L * B < 200 else 0, rng.choice([(8, 128), (4, 64), (2, 128)]), dtype, pages,
                 page_rows, lens)


# ---- lengths, page lists and values of a case -----------------------------------------------------------------------------------
def _lengths(case):
    """(rows of each utterance in its pages, rows of them that move)."""
    r = random.Random(case["lens"])
    if case["op"] == "attention":
        ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["B"])]
        return ctx, None
    rows = [r.randint(case["rows_lo"], case["rows_hi"]) for _ in range(case["B"])]
    return [n + r.randint(0, case["before"]) for n in rows], rows


def _index(values):
    return torch.tensor(values, dtype=torch.long, device=DEVICE)


def _table(case, ctx):
    """Pages of the utterances in some order among a few free ones; entries behind an utterance's last page are -1."""
    r, R = random.Random(case["lens"] + 1), case["page_rows"]
    need = [-(-n // R) for n in ctx]
    order = list(range(sum(need) + 3))
    r.shuffle(order)
    table, at = np.full((len(ctx), max(need)), -1, dtype=np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, len(order)


def _power(k):
    """2^k in 32 bits, k in -126 .. 127."""
    return ((k.int() + 127) << 23).view(torch.float32)


def _quantised(x, pages):
    """(codes, scales [..., ]) of rows x [..., hd]: the definition of the 8-bit types, elementary operations."""
    x = x.float()
    a = x.abs().amax(-1)
    if pages == "e4m3":
        m, e = torch.frexp(a)                                                            # a = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
        k = (e - 9 + (m > 0.875).int()).clamp(min=-126)
        code = (x * _power(-k)[..., None]).to(torch.float8_e4m3fn)
        return code, torch.where(a > 0, _power(k), 0.0)
    code = (x.double() * 127.0 / torch.where(a > 0, a, 1.0).double()[..., None]).round().to(torch.int8)
    return code, (a.double() / 127.0).float()


def _rows(g, dtype, *shape):
    """Rows as a decoder's projections leave them: normal, some elements much larger, each row of a magnitude of its own."""
    x = torch.randn(*shape, generator=g, device=DEVICE)
    x *= torch.exp(0.5 * torch.randn(*shape[:-1], 1, generator=g, device=DEVICE))
    x[..., ::29] *= 4.0
    return x.to(TYPES[dtype])


def _pool(g, case, L, n_pages):
    """Pages full of rows, each as the 8-bit types would hold it where the pages are of such a type."""
    shape = (L, n_pages, case["hkv"], case["page_rows"], case["hd"])
    s = {}
    for name in ("k", "v"):
        if case["pages"] in ("e4m3", "i8"):
            parts = [_quantised(_rows(g, "f32", *shape[1:]), case["pages"]) for _ in range(L)]
            s[name], s[name + "_scale"] = torch.stack([p[0].view(torch.uint8) for p in parts]).view(TYPES[case["pages"]]), torch.stack([p[1] for p in parts])
        else:
            s[name] = torch.stack([_rows(g, case["pages"], *shape[1:]) for _ in range(L)])
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    ctx, moved = _lengths(case)
    table, n_pages = _table(case, ctx)
    s = {"case": case, "table": torch.from_numpy(table).to(DEVICE), "ctx_len": torch.tensor(ctx, dtype=torch.int32, device=DEVICE), "max_ctx": max(ctx)}
    B, R, hkv, hd = case["B"], case["page_rows"], case["hkv"], case["hd"]
    if case["op"] == "attention":
        s["pool"] = _pool(g, case, 1, n_pages)
        s["q"] = (torch.randn(B, case["new"], case["hq"], hd, generator=g, device=DEVICE) * 1.5).to(TYPES[case["dtype"]])
        at, end = torch.arange(table.shape[1] * R, device=DEVICE), s["ctx_len"].long()[:, None]
        ends = end - (case["new"] - 1) + torch.arange(case["new"], device=DEVICE)                       # [B, new]
        s["seen"], s["stored"] = at < ends[..., None], at < end
        s["whole"] = s["table"].long().clamp(min=0)
        return s
    L = case["L"]
    # slots of the other cache: utterances in some order, the rows of a decoding step inside the packed projections of its tokens
    r, start, at = random.Random(case["lens"] + 2), [0] * B, 0
    order = list(range(B))
    r.shuffle(order)
    for b in order:
        start[b] = at
        at += moved[b] + r.randrange(3)
    utt = np.repeat(np.arange(B), moved)
    i = np.concatenate([np.arange(n) for n in moved])
    pos = np.array(ctx)[utt] - np.array(moved)[utt] + i
    s["slot"], s["page"], s["row"] = (torch.from_numpy(x.astype(np.int64)).to(DEVICE) for x in (np.array(start)[utt] + i, table[utt, pos // R], pos % R))
    s["start"], s["n_rows"] = (torch.tensor(v, dtype=torch.int32, device=DEVICE) for v in (start, moved))
    s["max_rows"] = max(moved)
    cache = _rows(g, case["dtype"], L, at, 3 * hkv, hd)
    s["cache_k"], s["cache_v"] = cache[:, :, hkv:2 * hkv], cache[:, :, 2 * hkv:]
    if case["op"] == "read":
        s["pool"] = _pool(g, case, L, n_pages)
    else:
        shape = (L, n_pages, hkv, R, hd)
        s["pool"] = {name: torch.zeros(shape, dtype=torch.uint8 if SIZE[case["pages"]] == 1 else TYPES[case["pages"]], device=DEVICE).view(TYPES[case["pages"]])
                     for name in ("k", "v")}
        if SIZE[case["pages"]] == 1:
            s["pool"] |= {name: torch.zeros(shape[:-1], device=DEVICE) for name in ("k_scale", "v_scale")}
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------------------
def _bytes(x):
    """Indexing and copies of 8-bit floats go by their bytes."""
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _plain_attention(s):
    c, pool = s["case"], s["pool"]
    B, hkv, hd, n, g = c["B"], c["hkv"], c["hd"], c["new"], c["hq"] // c["hkv"]

    def gathered(name):                                                                  # [B, hkv, rows, hd]
        x = _bytes(pool[name][0])[s["whole"]].view(pool[name].dtype).float()             # [B, pages, hkv, R, hd]
        if name + "_scale" in pool:
            x = x * pool[name + "_scale"][0][s["whole"]][..., None]
        return x.permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, hd)

    k = gathered("k").transpose(2, 3).contiguous()
    q = s["q"].float().view(B, n, hkv, g, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * g, hd)
    score = torch.matmul(q, k).view(B, hkv, n, g, -1) * (1.0 / math.sqrt(hd))
    score = score.masked_fill(~s["seen"][:, None, :, None], float("-inf"))
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)                                  # (of a token that sees nothing: finite)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total > 0, total, 1.0)).view(B, hkv, n * g, -1)
    v = gathered("v") * s["stored"][:, None, :, None]
    o = torch.matmul(p, v).view(B, hkv, n, g, hd).permute(0, 2, 1, 3, 4).reshape(B, n, c["hq"], hd)
    lse = torch.where(total > 0, top + torch.log(total), -math.inf)[..., 0].permute(0, 2, 1, 3).reshape(B, n, c["hq"])
    return {"out": o.to(s["q"].dtype), "lse": lse}


def _plain_write(s):
    c, pool = s["case"], s["pool"]
    for name in ("k", "v"):
        x = s["cache_" + name][:, s["slot"]]                                             # [L, rows, hkv, hd]
        if name + "_scale" in pool:
            x, scale = _quantised(x, c["pages"])
            pool[name + "_scale"][:, s["page"], :, s["row"]] = scale.transpose(0, 1)
        _bytes(pool[name])[:, s["page"], :, s["row"]] = _bytes(x).transpose(0, 1)
    return pool


def _plain_read(s):
    pool = s["pool"]
    for name in ("k", "v"):
        x = _bytes(pool[name])[:, s["page"], :, s["row"]].view(pool[name].dtype)         # [rows, L, hkv, hd]
        if name + "_scale" in pool:
            x = x.float() * pool[name + "_scale"][:, s["page"], :, s["row"]][..., None]
        s["cache_" + name][:, s["slot"]] = x.to(s["cache_" + name].dtype).transpose(0, 1)
    return {"k": s["cache_k"], "v": s["cache_v"]}


# ---- the framework's calls -----------------------------------------------------------------------------------------------------
_contexts = {}


def _context(s):
    """One context for the whole program, its workspace large enough for this state; the handle of the pages."""
    if "ctx" not in s:
        from paper_2603_11243_amd.binding import Context, KvPages
        c = s["case"]
        ctx = _contexts.setdefault(DEVICE, None) or Context(device=DEVICE)
        _contexts[DEVICE] = ctx
        if c["op"] == "attention":
            ctx.reserve(paged_utts=c["B"], paged_new=c["new"], paged_ctx=s["max_ctx"], paged_heads=(c["hq"], c["hkv"], c["hd"]))
        pool = s["pool"]
        s["ctx"], s["pages"] = ctx, KvPages(pool["k"], pool["v"], pool.get("k_scale"), pool.get("v_scale"))
    return s["ctx"], s["pages"]


def run(s):
    c = s["case"]
    if not own:
        return {"attention": _plain_attention, "write": _plain_write, "read": _plain_read}[c["op"]](s)
    ctx, pages = _context(s)
    if c["op"] == "attention":
        lse = torch.empty((c["B"], c["new"], c["hq"]), dtype=torch.float32, device=DEVICE)
        return {"out": ctx.paged_attention(s["q"], pages, s["table"], s["ctx_len"], max_ctx=s["max_ctx"], lse=lse), "lse": lse}
    call = ctx.kv_write_pages if c["op"] == "write" else ctx.kv_read_pages
    call(pages, s["table"], s["ctx_len"], s["cache_k"], s["cache_v"], start=s["start"], n_rows=s["n_rows"], max_rows=s["max_rows"], max_ctx=s["max_ctx"])
    return s["pool"] if c["op"] == "write" else {"k": s["cache_k"], "v": s["cache_v"]}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------------------
def work(case):
    ctx, moved = _lengths(case)
    es, ps, hd, B = SIZE[case["dtype"]], SIZE[case["pages"]], case["hd"], case["B"]
    row = hd * ps + (4 if ps == 1 else 0)                                                # of one head's K or V in pages
    entries = 4 * sum(-(-n // case["page_rows"]) for n in ctx) + 4 * B
    if case["op"] == "attention":
        pairs = sum(max(0, n - (case["new"] - 1 - t)) for n in ctx for t in range(case["new"]))
        queries = B * case["new"] * case["hq"]
        return {"bytes": 2 * sum(ctx) * case["hkv"] * row + 2 * queries * hd * es + 4 * queries + entries, "flops": 4 * pairs * case["hq"] * hd}
    n = 2 * case["L"] * sum(moved) * case["hkv"]
    return {"bytes": n * (row + hd * es) + entries + 8 * B, "flops": 3 * n * hd}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------------------
def _exact_power(k):
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_codes(x, pages):
    """Codes and scales of rows x [..., hd] in 64 bits."""
    a = x.abs().amax(-1)
    there = torch.where(a > 0, a, 1.0)
    if pages == "i8":
        return torch.round(x * 127.0 / there[..., None]), a / 127.0
    m, e = torch.frexp(there)
    k = torch.where(m > 448.0 / 512.0, e - 8, e - 9).clamp(min=-126)
    y = x * _exact_power(-k)[..., None]
    step = _exact_power(torch.frexp(y)[1].clamp(min=-5) - 4)                             # codes of 2^j .. 2^(j + 1) lie 2^(j - 3) apart, from j = -6 on
    return torch.round(y / step) * step, torch.where(a > 0, _exact_power(k), 0.0)


def exact(case, seed):
    s = prepare(case, seed)
    ctx, moved = _lengths(case)
    pool, R = s["pool"], case["page_rows"]
    table = s["table"].cpu().numpy()
    eight = SIZE[case["pages"]] == 1

    def stored(name, l, b, h, lo, hi):
        """Rows lo .. hi - 1 of utterance b."""
        pages = torch.from_numpy(table[b, lo // R:-(-hi // R)].astype(np.int64)).to(DEVICE)
        x = pool[name][l].view(torch.uint8)[pages, h].view(pool[name].dtype).double() if case["pages"] == "e4m3" else pool[name][l, pages, h].double()
        if eight:
            x = x * pool[name + "_scale"][l, pages, h].double()[..., None]
        first = lo // R * R
        return x.reshape(-1, case["hd"])[lo - first:hi - first]

    if case["op"] == "attention":
        g, n = case["hq"] // case["hkv"], case["new"]
        out = torch.zeros(case["B"], n, case["hq"], case["hd"], dtype=torch.float64, device=DEVICE)
        lse = torch.full((case["B"], n, case["hq"]), -math.inf, dtype=torch.float64, device=DEVICE)
        for b, total in enumerate(ctx):
            for h in range(case["hkv"]):
                k, v = stored("k", 0, b, h, 0, total), stored("v", 0, b, h, 0, total)
                for t in range(n):
                    end = total - (n - 1 - t)
                    if end > 0:
                        score = s["q"][b, t, h * g:(h + 1) * g].double() @ k[:end].T / math.sqrt(case["hd"])
                        lse[b, t, h * g:(h + 1) * g] = torch.logsumexp(score, -1)
                        out[b, t, h * g:(h + 1) * g] = torch.softmax(score, -1) @ v[:end]
        return {"out": out, "lse": lse}
    if case["op"] == "read":
        got = {name: s["cache_" + name].double() for name in ("k", "v")}
        for l in range(case["L"]):
            for b, n in enumerate(moved):
                a = int(s["start"][b])
                for h in range(case["hkv"]):
                    for name in ("k", "v"):
                        got[name][l, a:a + n, h] = stored(name, l, b, h, ctx[b] - n, ctx[b])
        return got
    got = {name: x.double() if x.dtype != torch.float8_e4m3fn else x.float().double() for name, x in pool.items()}
    for b, n in enumerate(moved):
        a, at = int(s["start"][b]), np.arange(ctx[b] - n, ctx[b])
        page, row = _index(table[b, at // R].tolist()), _index((at % R).tolist())
        for name in ("k", "v"):
            x = s["cache_" + name][:, a:a + n].double()                                  # [L, rows, hkv, hd]
            if eight:
                x, scale = _exact_codes(x, case["pages"])
                got[name + "_scale"][:, page, :, row] = scale.transpose(0, 1)
            got[name][:, page, :, row] = x.transpose(0, 1)
    if case["pages"] == "i8":
        got |= {name: got[name].to(torch.int8) for name in ("k", "v")}
    return got
