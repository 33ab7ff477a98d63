"""Two-phase batched decoding schedule of Sec. 3.2 around the library's calls (host-side policy only).

The paper sorts utterances by length, cuts them into batches under a token budget (50K tokens), batches the
CTC + LLM-verification pass separately from the auto-regressive fallback pass, and parks the acoustic embeddings
in host memory between the two.  `TwoPhaseDecoder.run` is that schedule:

  gate      ctc_gate over the whole batch (a streaming kernel without activations: no reason to cut it up)
  phase 1   verification bins planned with ssd_plan_batches on S + P + U of the utterances that failed the gate;
            per bin: ssd_select_unconfident -> verify_forward[_kv] -> accept_prefix
  between   mode "offload" (the paper's): the acoustic embeddings g of the rejected utterances are copied to pinned
            host memory and nothing else of phase 1 is kept; mode "resident": the K/V cache of phase 1 stays in HBM
            (what 288 GB make possible: a 50K-token batch of the 1B-class decoder is 4.9 GB of keys and values); mode
            "paged": the cache holds one bin, and behind each bin the rows of its rejected utterances go to pages, in 8 bits or as they are
            (which utterances those are is known on the device only: there are pages for the rows of all that are verified)
  phase 2   fallback bins planned on context length + steps of the rejected utterances; per bin, "offload" reloads g,
            re-runs the prompt [g; prompt; accepted prefix + the rejected token] with verify_forward_kv (whose greedy
            token at the rejected position is the first fallback token) and then ar_fallback; "resident" calls
            ar_fallback on the cached rows directly; "paged" reads them back from their pages first.

Everything numeric happens inside the library; this module only decides what goes into which call.  Copies between
device and pinned host memory are plain memcpys issued through torch on the context's stream.

`TreeFallback` is another phase 2: where a draft was rejected at one token, the tokens behind it are mostly still right, so
the fallback verifies them, at their place and shifted by one, as a tree behind the model's own token, several tokens a pass.
"""
from typing import List, Optional

import numpy as np
import torch

from .binding import Context, KvPages, plan_batches


class TreeFallback:
    """Continuation of rejected utterances by trees over their cached rows.  A round: the model's own next token with the rest of the draft behind
    it, once as if that token had replaced the draft's (substitution), once as if it had come before it (insertion) and once as if one more had been
    left out (deletion), common beginnings shared, goes through verify_tree; accept_tree keeps the longest branch whose tokens pass tau and moves its rows
    behind the context; the model's choice behind it begins the next round.  From tau 0.5 on a token that passes is the model's own choice, and the
    result that of ar_fallback up to the first near-tie: the two passes add in another order, and of two tokens whose likelihoods differ by no more
    than that either may be chosen.

    most_rows: contexts longer than that are cut between rounds by kv_evict to keep_rows rows (three quarters of it unless given): the first n_first and last
    n_recent ones stay, of the others those of the largest attention weight here.  They go to two caches of the fallback's own in turn; the rows
    of the attached one are only read, and it is attached again at the end."""

    def __init__(self, ctx: Context, max_utts: int, tau: float = 0.5, depth: int = 6, most_rows: Optional[int] = None, keep_rows: Optional[int] = None,
                 n_first: int = 4, n_recent: int = 32):
        self.ctx, self.tau, self.depth, self.most_rows, self.n_first, self.n_recent = ctx, tau, depth, most_rows, n_first, n_recent
        self.keep_rows = keep_rows if keep_rows is not None or most_rows is None else 3 * most_rows // 4
        assert depth >= 1 and (most_rows is None or n_first + n_recent <= self.keep_rows <= most_rows and self.keep_rows > 0)
        self.max_utts = max_utts
        self.room = 1 + 3 * depth                            # nodes of a tree at most
        self.own = [None, None]
        more = {}
        if most_rows is not None:
            self.slots = max_utts * (most_rows + 2 * self.room)
            more = {"evict_rows": self.slots, "evict_utts": max_utts, "evict_heads": (ctx.cfg.n_layers, ctx.cfg.n_kv_heads)}
        ctx.reserve(tree_nodes=max_utts * self.room, tree_utts=max_utts, **more)

    def _tree(self, token: int, draft, at: int, room: int):
        """(tokens, parents, draft positions behind each node) of the tree behind `token`, which stands where draft[at] was."""
        tokens, parent, follow, child = [token], [-1], [at + 1], {}
        for first in (at + 1, at, at + 2):
            node = 0
            for i in range(first, min(first + self.depth, len(draft))):
                key = (node, int(draft[i]))
                if key not in child:
                    if len(tokens) == room:
                        break
                    child[key] = len(tokens)
                    tokens.append(int(draft[i]))
                    parent.append(node)
                    follow.append(i + 1)
                node = child[key]
        return tokens, parent, follow

    def run(self, kv_start, ctx_len, first_tok, drafts: List[np.ndarray], n_steps: int) -> List[np.ndarray]:
        """kv_start, ctx_len: cached rows as for ar_fallback, with room for n_steps tokens and a tree behind them; first_tok (host): the model's own tokens at
        position ctx_len; drafts: the draft from the rejected token on.  Returns n_steps + 1 tokens an utterance, first_tok the first."""
        with torch.cuda.stream(self.ctx.stream):
            return self._run(kv_start, ctx_len, first_tok, drafts, n_steps)

    def _run(self, kv_start, ctx_len, first_tok, drafts, n_steps):
        ctx, dev = self.ctx, self.ctx.device
        start, length = np.array(kv_start, dtype=np.int32), np.array(ctx_len, dtype=np.int32)
        pos, done = length.copy(), [[] for _ in start]
        token, at = [int(t) for t in first_tok], [0] * len(start)
        k, _ = ctx.kv_tensors()
        mass = None if self.most_rows is None else torch.zeros((k.shape[0], k.shape[2], k.shape[1]), device=dev)
        before = ctx._kv, int(k.shape[1])
        assert len(start) <= self.max_utts
        try:
            self._rounds(start, length, pos, done, token, at, drafts, n_steps, mass)
        finally:
            if ctx._kv is not before[0]:
                ctx.attach_kv_cache(*before)
        return [np.array(d + [t], dtype=np.int32) for d, t in zip(done, token)]

    def _rounds(self, start, length, pos, done, token, at, drafts, n_steps, mass):
        """Adds n_steps tokens to every list of done; the other arrays follow."""
        ctx, dev, cuts = self.ctx, self.ctx.device, 0
        while True:
            live = [b for b in range(len(start)) if len(done[b]) < n_steps]
            if not live:
                break
            if mass is not None and any(done) and max(length[live]) > self.most_rows:
                mass = self._evict(live, start, length, mass, cuts % 2)
                cuts += 1
            trees = [self._tree(token[b], drafts[b], at[b], min(self.room, n_steps - len(done[b]))) for b in live]
            ids = torch.tensor([t for x in trees for t in x[0]], dtype=torch.int32, device=dev)
            cu, parent = np.cumsum([0] + [len(x[0]) for x in trees]), np.array([p for x in trees for p in x[1]])
            h = ctx.verify_tree(ids, cu, parent, start[live], length[live], pos0=pos[live], kv_mass=mass)
            acc = ctx.accept_tree(h, ids, cu, parent, self.tau, kv_start=start[live], ctx_len=length[live], kv_mass=mass)
            n, path, greedy = acc["accept_len"].tolist(), acc["path"].tolist(), acc["greedy_tok"].tolist()
            for i, b in enumerate(live):
                nodes = path[cu[i]:cu[i] + n[i]]
                done[b] += [trees[i][0][j] for j in nodes]
                length[b] += n[i]
                pos[b] += n[i]
                token[b], at[b] = greedy[cu[i] + nodes[-1]], trees[i][2][nodes[-1]]

    def _evict(self, live, start, length, mass, turn):
        """Cuts the live utterances into a cache of the fallback's own and attaches it; returns the weights of the rows there."""
        ctx = self.ctx
        k, v = ctx.kv_tensors()
        if self.own[turn] is None:
            self.own[turn] = torch.empty(ctx.kv_cache_bytes(self.slots), dtype=torch.uint8, device=ctx.device)
        k_out, v_out = ctx.kv_tensors(self.own[turn], self.slots)
        mass_out = torch.zeros((k.shape[0], k.shape[2], self.slots), device=ctx.device)
        keep = np.where(length[live] > self.most_rows, self.keep_rows, length[live])
        to = (np.arange(len(live)) * (self.most_rows + 2 * self.room)).astype(np.int32)
        ctx.kv_evict(k, v, mass, start[live], length[live], keep, self.n_first, self.n_recent, k_out, v_out, to, mass_out=mass_out)
        start[live], length[live] = to, keep
        ctx.attach_kv_cache(self.own[turn], self.slots)
        return mass_out


class TwoPhaseDecoder:
    def __init__(self, ctx: Context, wl, logits: torch.Tensor, cu_frames, ctc_to_llm: torch.Tensor,
                 speech_all: torch.Tensor, cu_speech_all, prompt_all: torch.Tensor, cu_prompt_all,
                 budget: int = 50000, mode: str = "resident", n_steps: int = 8, trees: Optional[dict] = None, pages_dtype: torch.dtype = torch.int8,
                 page_rows: int = 64):
        """trees: arguments of a TreeFallback (tau, depth, most_rows, ...) that continues the rejected utterances in place of ar_fallback.  pages_dtype, page_rows: of mode
        "paged" (int8, float8_e4m3fn, or the type of the cache, which keeps the rows as they are)."""
        assert mode in ("offload", "resident", "paged")
        self.pages: Optional[KvPages] = None
        self.pages_dtype, self.page_rows = pages_dtype, page_rows
        self.trees = None if trees is None else TreeFallback(ctx, len(cu_frames) - 1, **trees)
        self.room = n_steps + 2 + (0 if trees is None else self.trees.room)        # slots an utterance needs behind its rows
        self.ctx, self.wl, self.mode, self.budget, self.n_steps = ctx, wl, mode, int(budget), int(n_steps)
        self.logits, self.table = logits, ctc_to_llm
        self.cu_frames = np.ascontiguousarray(cu_frames, dtype=np.int32)
        self.speech_all, self.prompt_all = speech_all, prompt_all
        self.cu_s = np.ascontiguousarray(cu_speech_all, dtype=np.int32)
        self.cu_p = np.ascontiguousarray(cu_prompt_all, dtype=np.int32)
        self.B = len(self.cu_frames) - 1
        self.S, self.P, self.T = np.diff(self.cu_s), np.diff(self.cu_p), np.diff(self.cu_frames)
        dev, m = ctx.device, ctx.cfg
        n_frames, nS, nP = int(self.cu_frames[-1]), int(self.cu_s[-1]), int(self.cu_p[-1])
        # the largest bin is bounded by the budget, or by the longest utterance when that alone exceeds it
        longest = int((self.S + self.P + self.T).max()) + self.n_steps + 2
        cap = min(max(self.budget, longest), nS + nP + n_frames + self.B * (self.n_steps + 2))
        ctx.reserve(max_frames=n_frames, max_tokens=cap, max_verify_rows=min(cap, n_frames), max_utts=self.B,
                    ar_utts=self.B, ar_steps=self.n_steps)
        self.sel_buf = {"speech": torch.empty((min(cap, nS), m.d_model), dtype=speech_all.dtype, device=dev),
                        "prompt": torch.empty(min(cap, nP), dtype=torch.int32, device=dev),
                        "draft_ids": torch.empty(min(cap, n_frames), dtype=torch.int32, device=dev)}
        self.hv_buf = torch.empty((min(cap, n_frames), m.d_model), dtype=ctx.act_dtype, device=dev)
        # likelihoods and greedy tokens of every draft position of the batch, bins one after the other
        self.logp_all = torch.empty(n_frames, dtype=torch.float32, device=dev)
        self.greedy_all = torch.empty(n_frames, dtype=torch.int32, device=dev)
        self.gate_out = None
        # K/V slots: every verified utterance keeps its rows (resident), or one bin at a time (offload, paged)
        slots = (nS + nP + n_frames + self.B * self.room) if mode == "resident" else cap + self.B * self.room
        ctx.set_kv_cache(int(slots))
        self.kv_slots = int(slots)
        self.host_g: Optional[torch.Tensor] = None       # pinned staging for the acoustic embeddings (offload mode)
        if mode == "offload":
            self.host_g = torch.empty((nS, m.d_model), dtype=speech_all.dtype, pin_memory=True)
            self.dev_g = torch.empty((min(cap, nS), m.d_model), dtype=speech_all.dtype, device=dev)

    def _bins(self, lengths):
        return plan_batches(lengths, self.budget, padded=False) if len(lengths) else []

    def _page_lists(self, utts, rows):
        """Pages for so many rows of the utterances, one behind the other; [B, entries], -1 behind an utterance's last page."""
        need = -(-np.asarray(rows) // self.page_rows)
        if self.pages is None or self.pages.n_pages < need.sum():
            m = self.ctx.cfg
            self.pages = None                                # (the old ones go first)
            self.pages = KvPages.empty(int(need.sum()), self.page_rows, m.n_kv_heads, m.head_dim, self.pages_dtype, m.n_layers, self.ctx.device)
        lists = np.full((self.B, int(need.max())), -1, dtype=np.int32)
        for b, n, at in zip(utts, need, np.cumsum(need) - need):
            lists[b, :n] = np.arange(at, at + n)
        return lists

    def _starts(self, bins, rows):
        """First slots of the utterances of each bin, `room` behind the rows of each."""
        return [np.concatenate([[0], np.cumsum(rows[utts] + self.room)[:-1]]).astype(np.int32) for utts in bins]

    def _on_device(self, lists, bins, starts, rows):
        """(page lists, first slots, rows) of every bin.  One upload of each for all bins, while the stream has no work: a copy waits for what is queued before it."""
        utts, ends = np.concatenate(bins), np.cumsum([len(b) for b in bins])[:-1].tolist()
        parts = (torch.from_numpy(x).to(self.ctx.device).tensor_split(ends) for x in (lists[utts], np.concatenate(starts), rows[utts].astype(np.int32)))
        return list(zip(*parts))

    def _to_pages(self, place, most, acc):
        """The rows of a bin's rejected utterances, up to the end of their accepted prefixes, to their pages; lengths stay on the device."""
        (lists, start, before), (k, v) = place, self.ctx.kv_tensors()
        length = before + acc["accept_len"]
        moved = torch.where(acc["all_accepted"].bool(), 0, length).to(torch.int32)
        self.ctx.kv_write_pages(self.pages, lists, length, k, v, start=start, n_rows=moved, max_rows=most, max_ctx=most)

    def _from_pages(self, place, most):
        (lists, start, length), (k, v) = place, self.ctx.kv_tensors()
        self.ctx.kv_read_pages(self.pages, lists, length, k, v, start=start, n_rows=length, max_rows=most, max_ctx=most)

    def run(self, tau_slm: float) -> dict:
        with torch.cuda.stream(self.ctx.stream):             # what is copied to the host waits for the calls before it, whichever stream is current
            return self._run(tau_slm)

    def _run(self, tau_slm):
        ctx, wl, n_steps = self.ctx, self.wl, self.n_steps
        # ---- gate (Sec. 2.1) over everything
        g = ctx.ctc_gate(self.logits, self.cu_frames, wl.blank_id, wl.tau_ctc, out=self.gate_out)
        self.gate_out = g
        gate_pass = g["gate_pass"].cpu().numpy().astype(bool)
        draft_len = g["draft_len"].cpu().numpy()
        fail = np.flatnonzero(~gate_pass)
        res = {"gate_pass": gate_pass, "draft_len": draft_len, "accept_len": np.full(self.B, -1, np.int32),
               "tokens": {}, "verify_bins": 0, "fallback_bins": 0, "rejected": 0, "offloaded_bytes": 0}
        if len(fail) == 0:
            return res
        # ---- phase 1: verification bins (Sec. 2.2), longest first under the token budget
        n_rows = (self.S + self.P + draft_len)[fail]
        bins = [fail[b] for b in self._bins(n_rows)]
        res["verify_bins"] = len(bins)
        if self.mode == "paged":
            lists, starts = self._page_lists(fail, n_rows), self._starts(bins, self.S + self.P + draft_len)
            places = self._on_device(lists, bins, starts, self.S + self.P)
        kv_next = 0
        kv_start = np.zeros(self.B, np.int32)
        pending = []
        off = 0                                                # draft positions handed out so far
        goff = np.zeros(self.B, np.int64)                      # where an utterance's draft starts in logp_all / greedy_all
        for i, utts in enumerate(bins):
            sel = ctx.select_unconfident(utts, self.cu_frames, draft_len, g["draft_ctc"], self.table, self.speech_all,
                                         self.cu_s, self.prompt_all, self.cu_p, out=self.sel_buf)
            Mv = int(sel["cu_draft"][-1])
            ks = None
            if self.mode == "paged":
                ks = starts[i]
            elif self.mode == "resident":
                cap = (self.S + self.P + draft_len)[utts] + self.room
                ks = (kv_next + np.concatenate([[0], np.cumsum(cap)[:-1]])).astype(np.int32)
                kv_start[utts] = ks
                kv_next += int(cap.sum())
            hv = ctx.verify_forward(sel["speech"], sel["cu_speech"], sel["prompt"], sel["cu_prompt"], sel["draft_ids"],
                                    sel["cu_draft"], out=self.hv_buf[:Mv], kv_start=ks)
            acc = ctx.accept_prefix(hv, sel["draft_ids"], sel["cu_draft"], tau_slm,
                                    out={"draft_logp": self.logp_all[off:off + Mv], "greedy_tok": self.greedy_all[off:off + Mv],
                                         "accept_len": torch.empty(len(utts), dtype=torch.int32, device=ctx.device),
                                         "all_accepted": torch.empty(len(utts), dtype=torch.uint8, device=ctx.device)})
            if self.mode == "paged":
                self._to_pages(places[i], int((self.S + self.P + draft_len)[utts].max()), acc)
            goff[utts] = off + sel["cu_draft"][:-1]
            off += Mv
            pending.append((utts, acc))
        # one wait for the whole phase: prefix lengths decide who goes on
        for utts, acc in pending:
            res["accept_len"][utts] = acc["accept_len"].cpu().numpy()
        rej = np.array([b for b in fail if res["accept_len"][b] < draft_len[b]], dtype=np.int64)
        res["rejected"] = len(rej)
        if len(rej) == 0:
            return res
        A = res["accept_len"]
        # ---- between the phases
        if self.mode == "offload":
            with torch.cuda.stream(ctx.stream):
                for b in rej:                                  # g of the rejected utterances -> pinned host memory
                    lo, hi = int(self.cu_s[b]), int(self.cu_s[b + 1])
                    self.host_g[lo:hi].copy_(self.speech_all[lo:hi], non_blocking=True)
                    res["offloaded_bytes"] += (hi - lo) * self.speech_all.shape[1] * self.speech_all.element_size()
            ctx.stream.synchronize()                           # phase 1 is over; nothing of it stays on the device
        # ---- phase 2: fallback bins (Sec. 2.3) on context length + the tokens to come
        ctx_len_all = (self.S + self.P + A).astype(np.int32)
        fb_bins = [rej[b] for b in self._bins((ctx_len_all[rej] + n_steps + 2).astype(np.int32))]
        res["fallback_bins"] = len(fb_bins)
        outs = []
        if self.mode == "paged":
            starts = self._starts(fb_bins, ctx_len_all)
            places = self._on_device(lists, fb_bins, starts, ctx_len_all)
        for i, utts in enumerate(fb_bins):
            if self.mode != "offload":
                # the first fallback token is the model's own choice at the first rejected position
                first = ctx.gather_i32(self.greedy_all, goff[utts] + A[utts])
                ks, cl = kv_start[utts], ctx_len_all[utts]
                if self.mode == "paged":
                    ks = starts[i]
                    self._from_pages(places[i], int(cl.max()))
            else:
                # reload g, then re-run [g; prompt; accepted prefix + the rejected token] with the K/V cache on
                S_u = self.S[utts]
                cu_su = np.concatenate([[0], np.cumsum(S_u)]).astype(np.int32)
                with torch.cuda.stream(ctx.stream):
                    for k, b in enumerate(utts):
                        self.dev_g[int(cu_su[k]):int(cu_su[k + 1])].copy_(self.host_g[int(self.cu_s[b]):int(self.cu_s[b + 1])], non_blocking=True)
                re_len = draft_len.copy()
                re_len[utts] = A[utts] + 1
                sel = ctx.select_unconfident(utts, self.cu_frames, re_len, g["draft_ctc"], self.table, None,
                                             np.zeros(self.B + 1, np.int32), self.prompt_all, self.cu_p,
                                             out={"speech": self.sel_buf["speech"][:0], "prompt": self.sel_buf["prompt"],
                                                  "draft_ids": self.sel_buf["draft_ids"]}, d_model=int(self.speech_all.shape[1]),
                                             dtype=self.speech_all.dtype)
                cap = (self.S + self.P + A)[utts] + self.room
                ks = np.concatenate([[0], np.cumsum(cap)[:-1]]).astype(np.int32)
                cl = ctx_len_all[utts]
                Mv = int(sel["cu_draft"][-1])
                hv = ctx.verify_forward(self.dev_g[:int(cu_su[-1])], cu_su, sel["prompt"], sel["cu_prompt"], sel["draft_ids"],
                                        sel["cu_draft"], out=self.hv_buf[:Mv], kv_start=ks)
                acc = ctx.accept_prefix(hv, sel["draft_ids"], sel["cu_draft"], tau_slm, want_greedy=True)
                first = ctx.gather_i32(acc["greedy_tok"], sel["cu_draft"][1:] - 1)
            if self.trees is not None:
                f, ids, table = first.cpu().numpy(), g["draft_ctc"].cpu(), self.table.cpu()
                rest = [table[ids[self.cu_frames[b] + A[b]:self.cu_frames[b] + draft_len[b]].long()].numpy() for b in utts]
                for b, t in zip(utts, self.trees.run(ks, cl, f, rest, n_steps)):
                    res["tokens"][int(b)] = t
                continue
            toks = ctx.ar_fallback(ks, cl, first, n_steps)
            outs.append((utts, first, toks))
        for utts, first, toks in outs:
            f, t = first.cpu().numpy(), toks.cpu().numpy()
            for k, b in enumerate(utts):
                res["tokens"][int(b)] = np.concatenate([[f[k]], t[:, k]]).astype(np.int32)
        return res
