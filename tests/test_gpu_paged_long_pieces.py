"""paged_attention where a piece of a context is longer than the page numbers that a wavefront holds at a time (4096 rows), against 64 bits."""
import numpy as np
import pytest
import torch

from pages import EIGHT, TYPE
from paper_2603_11243_amd.binding import Context, KvPages

pytestmark = pytest.mark.gpu

PAIRS = [("f16", "f16"), ("bf16", "bf16"), ("f32", "f32"), ("f16", "e4m3"), ("bf16", "i8"), ("f32", "i8"), ("f32", "e4m3")]


def _case(pair, hd, lens, page_rows, seed=0):
    """Pages of one K/V head in any order, the rows behind an utterance's last one NaN; values [pages, rows, head_dim] in 64 bits beside them."""
    g, r = torch.Generator(device="cuda").manual_seed(seed), np.random.default_rng(seed)
    need = [-(-n // page_rows) for n in lens]
    n_pages = sum(need) + 3
    order, at = r.permutation(n_pages), 0
    table = np.full((len(lens), max(need)), -1, dtype=np.int32)
    used = np.zeros((n_pages, page_rows), dtype=bool)
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
        j = np.arange(lens[b])
        used[table[b, j // page_rows], j % page_rows] = True
    used = torch.from_numpy(used).cuda()
    parts, value = [], []
    for _ in range(2):
        x = torch.randn(n_pages, page_rows, hd, generator=g, device="cuda")
        if pair[1] in EIGHT:
            code = (x * 40).to(TYPE[pair[1]])
            scale = torch.exp(0.5 * torch.randn(n_pages, page_rows, generator=g, device="cuda")) / 40
            value.append(code.float().double() * scale.double()[..., None])
            parts.append((code[:, None].contiguous(), torch.where(used, scale, float("nan"))[:, None].contiguous()))
        else:
            x = (x * torch.exp(0.5 * torch.randn(n_pages, page_rows, 1, generator=g, device="cuda"))).to(TYPE[pair[1]])
            value.append(x.double())
            parts.append((x.masked_fill(~used[..., None], float("nan"))[:, None].contiguous(), None))
    (k, ks), (v, vs) = parts
    return KvPages(k, v, ks, vs), value, table


def _run(pair, hd, hq, n_new, lens, page_rows, bad=()):
    """bad: (utterance, entry) of pages that are none.  The bound is that of pages.attention with the sums as they are cut: a wavefront adds the 32 rows of one of four
    blocks of a piece, `blocks` of them one after the other, each as up to three products."""
    B = len(lens)
    pages, (kd, vd), table = _case(pair, hd, lens, page_rows)
    c = Context(device="cuda:0")
    c.reserve(paged_utts=B, paged_new=n_new, paged_ctx=table.shape[1] * page_rows, paged_heads=(hq, 1, hd))
    q = (torch.randn(B, n_new, hq, hd, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)) * 1.5).to(TYPE[pair[0]])
    lost = table.copy()
    for b, e in bad:
        lost[b, e] = -7
    lse = torch.empty(B, n_new, hq, device="cuda")
    c.device_flags()
    out = c.paged_attention(q, pages, torch.from_numpy(lost).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), lse=lse)
    assert c.device_flags() == (4 if bad else 0)
    u, eight, three = torch.finfo(q.dtype).eps / 2, pair[1] in EIGHT, pair[0] == "f32"
    left = (2.0 ** -24 if three else 2.0 ** -17) if eight else {"f16": 2.0 ** -22, "bf16": 2.0 ** -17, "f32": 0}[pair[1]]
    blocks = -(-max(lens) // 128)                            # (of a context in one piece; more pieces are shorter)
    for b, n in enumerate(lens):
        j = torch.arange(n, device="cuda")
        entry = torch.from_numpy(lost[b]).cuda().long()[j // page_rows]
        seen = entry >= 0
        k, v = kd[entry.clamp(min=0), j % page_rows], vd[entry.clamp(min=0), j % page_rows]
        for t in range(n_new):
            here = seen & (j < n - (n_new - 1 - t))
            kk, vv, x = k[here], v[here], q[b, t].double()
            s = x @ kk.T.contiguous() * hd ** -0.5
            d = ((3 if three else 2) * hd + 8) * 2.0 ** -24 * hd ** -0.5 * (x.abs() @ kk.abs().T.contiguous()).amax(1)
            p = torch.exp(s - s.amax(1, keepdim=True))
            total = p.sum(1)
            p /= total[:, None]
            sums = 2 * d + 2.0 ** -22 + (96 * blocks + 64) * 2.0 ** -24
            want, spread = p @ vv, p @ vv.abs()
            tol = u * want.abs() + (left + sums)[:, None] * (1 + u) * spread + u * torch.finfo(q.dtype).tiny + 2.0 ** -30 * (pair[1] == "f16")
            assert (out[b, t].double() - want).abs().le(tol).all(), (b, t, ((out[b, t].double() - want).abs() / tol).max())
            want = s.amax(1) + torch.log(total)
            assert (lse[b, t].double() - want).abs().le(sums + 2.0 ** -22 * want.abs()).all(), (b, t)
    c.close()


@pytest.mark.parametrize("pair", PAIRS)
@pytest.mark.parametrize("hd, hq, n_new, page_rows", [(64, 512, 2, 64), (128, 512, 1, 256), (64, 272, 1, 16)])
def test_pieces_longer_than_the_pages_known_at_a_time(pair, hd, hq, n_new, page_rows):
    """So many tiles of query rows that few pieces run at once: two contexts of 70000 rows are some 16 pieces of 8000 rows."""
    _run(pair, hd, hq, n_new, [70000, 66001], page_rows)


@pytest.mark.parametrize("pair", [("f16", "f16"), ("bf16", "i8"), ("f32", "f32")])
def test_pages_that_are_none_far_inside_a_piece(pair):
    """Also the first and the last page that are found later than the others, and all from one on."""
    _run(pair, 64, 512, 2, [70000, 40000], 64, bad=[(0, 64), (0, 127), (0, 128), (0, 700), (1, 63), (1, 129)] + [(1, e) for e in range(400, 625)])


def test_more_utterances_than_pieces_at_once():
    _run(("bf16", "e4m3"), 64, 512, 1, [9000] * 30 + [1, 40000], 64)
