"""K/V rows in pages for the tests: page lists, the 8-bit types by their definitions in 64 bits, attention of the newest tokens in 64 bits."""
import numpy as np
import torch

TYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
EIGHT = ("e4m3", "i8")


def code_values():
    """The values of the 256 codes of e4m3: sign, 4 exponent bits biased by 7, 3 fraction bits; all ones is NaN."""
    v = []
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        x = np.nan if c & 127 == 127 else f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        v.append(-x if c & 128 else x)
    return np.array(v)


def to_e4m3(y):
    """Nearest e4m3 value, halves to the even code (|y| <= 448, float64)."""
    step = 2.0 ** (np.maximum(np.frexp(y)[1] - 1, -6) - 3.0)
    return np.rint(y / step) * step


def quantised(x, kind):
    """(values of the codes, scales) of rows x [.., head_dim]."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        a = np.abs(x).max(-1)
        odd = ~np.isfinite(x).all(-1)
        a = np.where(odd, 0.0, a)
        x = np.where(odd[..., None], 0.0, x)
        if kind == "e4m3":
            m, e = np.frexp(a)
            k = np.maximum(np.where(m > 0.875, e - 8, e - 9), -126)
            scale, code = np.where(a > 0, 2.0 ** k, 0.0), to_e4m3(x * 2.0 ** -k[..., None].astype(float))
            code = np.where(k[..., None] == 120, np.clip(code, -240, 240), code)      # 256 would be worth 2^128
        else:
            scale = (a / 127).astype(np.float32).astype(np.float64)
            scale = np.where(scale * 127 >= 2.0 ** 128 - 2.0 ** 103, np.nextafter(scale.astype(np.float32), np.float32(0)), scale)
            code = np.rint(x * 127 / np.where(a > 0, a, 1)[..., None])
    return code, np.where(odd, np.nan, scale)


def numpy64(t):
    return t.double().cpu().numpy() if t.dtype != torch.float8_e4m3fn else code_values()[t.view(torch.uint8).cpu().numpy()]


class Pool:
    """Pages of B utterances of ctx_len rows in some order among free ones; everything that is no row of an utterance holds NaN (as a code, a value or a scale), and
    entries behind an utterance's last page are numbers of no page."""

    def __init__(self, kind, heads, ctx_len, page_rows, seed=0, layers=1, spare=2, most=None):
        H, hd = heads
        g, r = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        self.kind, self.page_rows, self.H, self.hd, self.layers = kind, page_rows, H, hd, layers
        need = [-(-n // page_rows) for n in ctx_len]
        entries = -(-(most or max(ctx_len)) // page_rows)
        order, at = r.permutation(sum(need) + spare), 0
        table = r.choice([-1, -7, 1 << 30, -2 ** 31], size=(len(ctx_len), entries)).astype(np.int32)
        self.n_pages = len(order)
        self.used = np.zeros((self.n_pages, page_rows), dtype=bool)
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
            for j in range(ctx_len[b]):
                self.used[table[b, j // page_rows], j % page_rows] = True
        self.table_host, self.ctx_host = table, np.array(ctx_len, dtype=np.int32)
        self.table, self.ctx_len = torch.from_numpy(table).cuda(), torch.tensor(ctx_len, dtype=torch.int32).cuda()
        shape = (layers, self.n_pages, H, page_rows, hd)
        used = torch.from_numpy(self.used)[None, :, None, :]
        self.parts = {}
        for name in ("k", "v"):
            x = torch.randn(shape, generator=g) * torch.exp(0.5 * torch.randn(shape[:-1], generator=g))[..., None]
            if kind in EIGHT:
                code, scale = quantised(x.numpy(), kind)
                code = torch.from_numpy(code).float().to(TYPE[kind])
                if kind == "e4m3":
                    code.view(torch.uint8)[~used.expand(shape[:-1])] = 127
                scale = torch.from_numpy(scale.astype(np.float32))
                scale[~used.expand(shape[:-1])] = float("nan")
                self.parts[name], self.parts[name + "_scale"] = code.cuda(), scale.cuda()
            else:
                x = x.to(TYPE[kind])
                x[~used.expand(shape[:-1])] = float("nan")
                self.parts[name] = x.cuda()

    def pages(self):
        from paper_2603_11243_amd.binding import KvPages
        return KvPages(self.parts["k"], self.parts["v"], self.parts.get("k_scale"), self.parts.get("v_scale"))

    def value(self, name):
        """[layers, pages, heads, rows, head_dim] in 64 bits."""
        x = numpy64(self.parts[name])
        return x * numpy64(self.parts[name + "_scale"])[..., None] if self.kind in EIGHT else x

    def rows(self, value, b, n=None):
        """Rows 0 .. n - 1 of utterance b: [layers, n, heads, head_dim]."""
        j = np.arange(self.ctx_host[b] if n is None else n)
        return value[:, self.table_host[b, j // self.page_rows], :, j % self.page_rows].transpose(1, 0, 2, 3)


def attention(q, pool, n_new, scale=None, lost=lambda b, j: False):
    """(out, its bound, lse, its bound) of q [B, n_new, query heads, head_dim] in 64 bits; lost(b, j): rows in bad pages.
    u: half a step of q's type.  Operands of the first product are q in as many 16-bit values as hold it exactly (1 bfloat16, 2 half with 8-bit pages, 3 fp32) and exact
    codes: c hd products added in fp32, off by at most (c hd + 8) 2^-24 sum |q k| |scale| =: d, scale of the row, scaling and the factor to base 2 among the 8.
    A weight: 2 d (its own score and the sum), the exponential's 2^-22, and what its values of 16 bits leave: half 2^-22 (and of what is below 2^-17 of the largest 2^-40
    of that), bfloat16 2^-17, three 2^-24; fp32 none.  Sums over n keys in fp32, as many products as there are values: 3 n 2^-24 of what is added, the joining a few more.  The output is rounded once:
    by u relative to it, and of subnormal results (of half below 2^-14, 2^-24 apart) by half of that step, eps * tiny / 2."""
    B, _, Hq, hd = q.shape
    scale = hd ** -0.5 if scale is None else scale
    u = torch.finfo(q.dtype).eps / 2
    eight = pool.kind in EIGHT
    c = 3 if q.dtype == torch.float32 else 2
    left = (2.0 ** -24 if q.dtype == torch.float32 else 2.0 ** -17) if eight else {"f16": 2.0 ** -22, "bf16": 2.0 ** -17, "f32": 0}[pool.kind]
    floor = 2.0 ** -40 if pool.kind == "f16" else 0
    k, v = pool.value("k"), pool.value("v")
    qq = q.double().cpu().numpy()
    out, tol = np.zeros(qq.shape), np.zeros(qq.shape)
    lse, lse_tol = np.full(qq.shape[:3], -np.inf), np.zeros(qq.shape[:3])
    group = Hq // pool.H
    for b in range(B):
        kb, vb = pool.rows(k, b)[0], pool.rows(v, b)[0]
        there = np.array([not lost(b, j) for j in range(len(kb))], dtype=bool)
        for t in range(n_new):
            n = max(0, int(pool.ctx_host[b]) - (n_new - 1 - t))
            seen = np.flatnonzero(there[:n])
            if not len(seen):
                continue
            for h in range(Hq):
                kk, vv, x = kb[seen, h // group], vb[seen, h // group], qq[b, t, h]
                s = kk @ x * scale
                d = (c * hd + 8) * 2.0 ** -24 * abs(scale) * (abs(kk) @ abs(x)).max()
                top = s.max()
                p = np.exp(s - top)
                l = p.sum()
                p /= l
                sums = 2 * d + 2.0 ** -22 + (3 * n + 32) * 2.0 ** -24
                out[b, t, h] = p @ vv
                tol[b, t, h] = u * abs(out[b, t, h]) + (1 + u) * ((left + sums) * (p @ abs(vv)) + floor * abs(vv).sum(0)) + u * torch.finfo(q.dtype).tiny + 2.0 ** -100
                lse[b, t, h] = top + np.log(l)
                lse_tol[b, t, h] = sums + 2.0 ** -22 * abs(lse[b, t, h])
    return out, tol, lse, lse_tol
