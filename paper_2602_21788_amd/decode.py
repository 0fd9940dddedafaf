"""Answering with a model that was trained with this library's attention: new tokens of many sequences over a paged 8-bit cache, wired from the C-ABI calls.

Only buffers and tables live here (which pages a sequence owns, how long it is, which position comes next); every step of the path runs in the library's own kernels:
  fcp_rotary -> fcp_cache_append -> fcp_cache_attn (weigh) for new tokens; fcp_attn_fwd_step_direct for prompts, whose keys then go into the cache and whose
  weights fcp_cache_weigh adds up; fcp_cache_evict when a sequence outgrows its budget.
Several continuations of every prompt (BeamDecoder):
  fcp_beam_select -> fcp_cache_fork -> fcp_rotary -> fcp_cache_append -> fcp_cache_attn_shared; fcp_cache_compact when the pool is to shrink.

    python -m paper_2602_21788_amd.decode        # a small run: prompts, tokens, eviction; beams
"""
from __future__ import annotations

from contextlib import contextmanager

import numpy as np
import torch

from . import binding as B
from .rank import RankAttention

FORMATS = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


class CacheDecoder:
    """Sequences 0 .. n_seqs - 1 of one layer.  rot_dim: channels of a head that turn with the position (0: none); turns: what fcp_rotary_frequencies gives."""

    def __init__(self, n_seqs, n_pages, max_pages, hq, hkv, head_dim, page_tokens=64, fmt="e4m3", rot_dim=None, turns=None, layout=B.FCP_ROTARY_HALF,
                 magnitude=1.0, softmax_scale=None, device="cuda:0"):
        dev = self.device = torch.device(device)
        self.hq, self.hkv, self.D, self.P = hq, hkv, head_dim, page_tokens
        self.scale = float(softmax_scale) if softmax_scale is not None else 1.0 / float(np.sqrt(head_dim))
        mk = lambda *s: torch.zeros(*s, dtype=torch.int8, device=dev).view(FORMATS[fmt])
        ones = lambda: torch.ones(n_pages, hkv, device=dev)
        self.cache = B.Cache(mk(n_pages, hkv, page_tokens, head_dim), mk(n_pages, hkv, page_tokens // 16, head_dim, 16), ones(), ones(),
                             torch.zeros(n_pages, hkv, page_tokens, device=dev))
        self.rot_dim, self.layout, self.magnitude = head_dim if rot_dim is None else rot_dim, layout, magnitude
        if self.rot_dim:
            turns = B.fcp_rotary_frequencies(self.rot_dim)[0] if turns is None else turns
            self.turns = torch.as_tensor(turns, dtype=torch.float64).to(dev)
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages = np.full((n_seqs, max_pages), -1, np.int32)
        self.kv_len = np.zeros(n_seqs, np.int32)             # cached tokens
        self.next_pos = np.zeros(n_seqs, np.int64)           # position of the next token: evicted ones still count
        self._scratch = {}

    # -- tables ------------------------------------------------------------------------------------------------------------
    def _to(self, a):
        return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(self.device)

    def _upload(self):
        self.pages_d, self.kv_len_d = self._to(self.pages), self._to(self.kv_len)

    def _work(self, which, tq=0):
        """Work space of the largest call so far of a kind."""
        n = B.fcp_cache_scratch_bytes(which, self.cache, *self.pages.shape, tq, self.hq)
        if which not in self._scratch or self._scratch[which].numel() < n:
            self._scratch[which] = torch.empty(n, dtype=torch.uint8, device=self.device)
        return self._scratch[which]

    def _counts(self, news):
        news = np.asarray(news, np.int32)
        if news.shape != self.kv_len.shape or (news < 0).any():
            raise ValueError("a number of tokens, 0 or more, is needed for every sequence")
        return news

    def _fit(self, q, k, v, rows, whole=False):
        """Refuses rows that a call of the path would refuse, before pages change hands.  whole: nothing between rows, as prompts' attention takes them."""
        for name, x, h in (("q", q, self.hq), ("k", k, self.hkv), ("v", v, self.hkv)):
            at, row = B._rows(x, h, self.D, name)
            if x.shape[0] != rows:
                raise ValueError(f"{name} must have {rows} rows, one for each new token")
            if x.device != self.cache.k.device or row < h * self.D or row % 8 or at % 16 or (whole and not x.is_contiguous()):
                raise ValueError(f"{name} must be on the cache's device, 16-byte aligned, {'contiguous' if whole else 'its rows a multiple of 8 elements apart'}")

    @contextmanager
    def _grown(self, news):
        """Room for news[s] more tokens of every sequence: (cu_seqlens, positions) of the new rows.  Where something fails inside, the tables are as they were."""
        need = [-(-(int(n) + int(m)) // self.P) - int((row >= 0).sum()) for n, m, row in zip(self.kv_len, news, self.pages)]
        if sum(max(n, 0) for n in need) > len(self.free) or (self.kv_len + news > self.pages.shape[1] * self.P).any():
            raise MemoryError("no page left: evict, or close a sequence")
        taken = []
        for s, n in enumerate(need):
            at = int((self.pages[s] >= 0).sum())
            for i in range(n):
                self.pages[s, at + i] = self.free.pop()
                taken.append((s, at + i))
        pos = np.concatenate([np.arange(p, p + m) for p, m in zip(self.next_pos, news)]) if sum(news) else np.zeros(0)
        self.kv_len += news
        self.next_pos += news
        try:
            self._upload()
            yield self._to(np.concatenate([[0], np.cumsum(news)])), self._to(pos)
        except BaseException:
            for at in reversed(taken):
                self.free.append(int(self.pages[at]))
                self.pages[at] = -1
            self.kv_len -= news
            self.next_pos -= news
            raise

    def close(self, seq):
        """Forgets a sequence; its pages are free."""
        self.free += [int(p) for p in self.pages[seq] if p >= 0]
        self.pages[seq], self.kv_len[seq], self.next_pos[seq] = -1, 0, 0

    def _rotate(self, q, k, pos):
        if self.rot_dim:
            B.fcp_rotary([(q, q, pos), (k, k, pos)], self.turns, self.rot_dim, self.layout, self.magnitude)

    # -- the path ----------------------------------------------------------------------------------------------------------
    def prefill(self, q, k, v, lens):
        """Prompts of lens[s] tokens for empty sequences: bf16 rows q [sum, hq, D], k, v [sum, hkv, D] (turned in place).  Returns O [sum, hq, D], LSE [hq, sum].
        O and LSE are those of the keys and values as given.  The cached tokens' weights are exp(score - LSE) with the scores of the cached, 8-bit keys: a row's add up to 1 but for the keys'
        rounding."""
        lens = self._counts(lens)
        self._fit(q, k, v, int(lens.sum()), whole=True)
        if self.kv_len.any():
            raise ValueError("prefill is for empty sequences; step() takes the next piece of a prompt")
        some = lens[lens > 0]
        if not len(some):
            return torch.empty_like(q), torch.empty(self.hq, 0, dtype=torch.float32, device=self.device)
        ra = RankAttention(some, np.ones(len(some), np.int32), 0, self.hq, self.hkv, self.D, self.scale, device=self.device)
        ra.q, ra.k, ra.v, ra.d_o = q, k, v, None
        ra._alloc_outputs()
        with self._grown(lens) as (cu, pos):
            self._rotate(q, k, pos)
            ra.forward_direct()
            B.fcp_cache_append(self.cache, k, v, cu, self.kv_len_d, self.pages_d)
            B.fcp_cache_weigh(self.cache, q, ra.lse, cu, self.kv_len_d, self.pages_d, self.scale)
        return ra.o, ra.lse

    def step(self, q, k, v, news, weigh=True):
        """news[s] new tokens of every sequence (0, 1, or more): bf16 rows as in prefill.  Returns O [sum, hq, D], LSE [hq, sum]."""
        news = self._counts(news)
        self._fit(q, k, v, int(news.sum()))
        o = torch.empty(q.shape, dtype=torch.bfloat16, device=self.device)
        lse = torch.empty(q.shape[1], q.shape[0], dtype=torch.float32, device=self.device)
        which = B.FCP_SCRATCH_CACHE_WEIGH if weigh else B.FCP_SCRATCH_CACHE_ATTN
        scratch = self._work(which, q.shape[0])
        with self._grown(news) as (cu, pos):
            self._rotate(q, k, pos)
            B.fcp_cache_append(self.cache, k, v, cu, self.kv_len_d, self.pages_d)
            B.fcp_cache_attn(self.cache, q, cu, self.kv_len_d, self.pages_d, self.scale, o, lse, scratch, weigh=weigh)
        return o, lse

    def evict(self, budget, n_first=4, n_recent=64):
        """Cuts every sequence to `budget` tokens; the old pages are free.  Returns the kept token numbers [n_seqs, hkv, budget] (-1 past the last)."""
        if budget < max(1, n_first + n_recent) or min(n_first, n_recent) < 0:
            raise ValueError("budget must be at least 1 and n_first + n_recent, which must not be negative")
        self._upload()
        new_len = np.minimum(self.kv_len, budget).astype(np.int32)
        counts = -(-new_len // self.P)
        width = max(-(-min(budget, self.pages.shape[1] * self.P) // self.P), 1)
        if counts.sum() > len(self.free):
            raise MemoryError("eviction moves tokens to new pages, and there are too few")
        new_pages = np.full((len(new_len), width), -1, np.int32)
        taken = 0
        for s, n in enumerate(counts):
            for i in range(n):
                taken += 1
                new_pages[s, i] = self.free[-taken]
        kept = torch.empty(len(new_len), self.hkv, budget, dtype=torch.int32, device=self.device)
        B.fcp_cache_evict(self.cache, self.pages_d, self.kv_len_d, self._to(new_pages), budget, n_first, n_recent, kept,
                          torch.empty(len(new_len), dtype=torch.int32, device=self.device), self._work(B.FCP_SCRATCH_CACHE_EVICT))
        self.free = self.free[: len(self.free) - taken] + [int(p) for p in self.pages[self.pages >= 0]]
        self.pages[:] = -1
        self.pages[:, :width] = new_pages[:, : self.pages.shape[1]]
        self.kv_len = new_len
        self._upload()
        return kept


class BeamDecoder:
    """`beams` continuations of each of n_prompts prompts, one layer.  The tables live on the device: a step needs nothing from the host but the rows, and the host waits for it only to learn whether
    there were pages enough (check).

        dec.prefill(q, k, v, lens)                      # the prompts
        loop: tokens, parents = dec.select(logits)      # logits [n_prompts, vocab] after the prompts, then [n_prompts * beams, vocab]
              o, lse = dec.step(q, k, v)                # the rows of these tokens, one for each beam
        dec.sequences()                                 # what each beam says
    """

    def __init__(self, n_prompts, beams, n_pages, max_pages, hq, hkv, head_dim, end_token=-1, **kw):
        self.prompts = CacheDecoder(n_prompts, n_pages, max_pages, hq, hkv, head_dim, **kw)
        self.n, self.beams, self.end = n_prompts, beams, end_token
        self.cache, self.device, self.scale = self.prompts.cache, self.prompts.device, self.prompts.scale
        i32 = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=self.device)
        rows = n_prompts * beams
        self._tables = [(i32(rows, max_pages), i32(rows)) for _ in range(2)]           # this step's and the next one's, in turn
        self.counts = i32(3)
        up = self.prompts._to
        self._ones, self._none, self._cu, self._groups = up(np.ones(rows)), up(np.zeros((1, 1))), up(np.arange(rows + 1)), up(np.arange(n_prompts + 1) * beams)
        self._fork_scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_FORK, self.cache, rows, max_pages), dtype=torch.uint8, device=self.device)
        self._attn_scratch = torch.empty(B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_SHARED, self.cache, rows, max_pages, rows, hq), dtype=torch.uint8, device=self.device)
        self._beam_scratch = None

    def prefill(self, q, k, v, lens):
        """The prompts, as CacheDecoder.prefill."""
        out = self.prompts.prefill(q, k, v, lens)
        self.prompts._upload()                               # (prompts may all be empty)
        self.pages, self.kv_len = self.prompts.pages_d, self.prompts.kv_len_d
        self._lens = np.asarray(lens, np.int64)
        self._longest = int(np.max(lens, initial=0))         # tokens of the longest sequence that goes on, or more
        self._shared = self.prompts._to(np.asarray(lens) // self.prompts.P * self.prompts.P)     # (the page in which a prompt ends is every beam's own)
        self.score, self.done = torch.zeros(self.n, device=self.device), torch.zeros(self.n, dtype=torch.uint8, device=self.device)
        self.chosen, self.history, self.steps = None, [], 0
        self._unchecked = False                              # whether a step may have found too few pages
        return out

    def select(self, logits):
        """The best tokens behind the beams so far: (tokens, parents) [n_prompts, beams], best first; parents are rows of the logits, -1 where there is no candidate.  self.score, self.done follow."""
        if self.chosen is not None:
            raise ValueError("step() takes the rows of the tokens that were chosen before the next ones are")
        width = 1 if not self.history else self.beams
        mk = lambda dt: torch.empty(self.n, self.beams, dtype=dt, device=self.device)
        parent, token, score, done = mk(torch.int32), mk(torch.int32), mk(torch.float32), mk(torch.uint8)
        n = B.fcp_beam_scratch_bytes(self.n, width, logits.shape[1], self.beams)
        if self._beam_scratch is None or self._beam_scratch.numel() < n:
            self._beam_scratch = torch.empty(n, dtype=torch.uint8, device=self.device)
        B.fcp_beam_select(logits, self.score, width, parent, token, score, self._beam_scratch, self.done, self.end, done)
        self.score, self.done, self.chosen = score.view(-1), done.view(-1), parent.view(-1)
        self.history.append((parent, token))
        return token, parent

    def _over(self):
        """[n_prompts, 1] bool: prompts of which no chosen beam goes on: they have all ended, or there was no candidate.  This stays so."""
        return torch.logical_or(self.done, self.chosen < 0).view(self.n, self.beams).all(1, keepdim=True)

    def step(self, q, k, v, check=True):
        """The rows of the chosen tokens, bf16 [n_prompts * beams, heads, D] (turned in place): O, LSE.  check: raises MemoryError, and leaves the beams as they were, where the pool has too few
        pages, or a new token would go into one that was lacking in an earlier step; the host waits for this.  Without it tokens that found no page are seen by nobody, and if the page would
        have been a copy of one that is begun, neither are the beam's earlier tokens in it nor its next ones, until that page ends.
        Prompts whose beams have all ended stay as they are: their rows are not appended and take no pages, O is 0 and LSE -inf for them.  (With an end token this takes 5 small launches, some 18 us
        of a step of 16 prompts' 8 beams that takes 89 without.)"""
        if self.chosen is None:
            raise ValueError("select() chooses the tokens whose rows step() takes")
        dec, rows = self.prompts, self.n * self.beams
        dec._fit(q, k, v, rows)
        if self._longest == dec.pages.shape[1] * dec.P:      # (the host waits here alone: prompts may have ended)
            self._longest = int(np.max(self._lens[~self._over().cpu().numpy()[:, 0]] + self.steps, initial=0))
            if self._longest == dec.pages.shape[1] * dec.P:
                raise MemoryError("a sequence's table is full")
        o, lse = torch.empty(q.shape, dtype=torch.bfloat16, device=self.device), torch.empty(dec.hq, rows, dtype=torch.float32, device=self.device)
        pages, kv_len = self._tables[self.steps % 2]
        news = self._ones if self.end < 0 else torch.where(self._over(), self._none, self._ones.view(self.n, self.beams)).view(-1)
        B.fcp_cache_fork(self.cache, self.pages, self.kv_len, self.chosen, news, pages, kv_len, self.counts, self._fork_scratch)
        if check and int(self.counts[1]):
            raise MemoryError("no page left")
        if check and self._unchecked and bool(((pages.gather(1, (kv_len - 1).clamp(min=0).long()[:, None] // dec.P)[:, 0] < 0) & (news > 0)).any()):
            raise MemoryError("a beam has no page for its next token: an earlier step without check found none")
        if dec.rot_dim:
            dec._rotate(q, k, kv_len - 1)                    # (the new token is the last one)
        tokens = kv_len if self.end < 0 else kv_len * news   # (a row of a sequence of no tokens is not appended, and sees nothing)
        B.fcp_cache_append(self.cache, k, v, self._cu, tokens, pages)
        B.fcp_cache_attn_shared(self.cache, q, self._cu, tokens, pages, self._groups, self._shared, self.scale, o, lse, self._attn_scratch)
        self.pages, self.kv_len, self.chosen = pages, kv_len, None
        self._unchecked |= not check
        self.steps += 1
        self._longest += 1
        return o, lse

    def compact(self):
        """Moves the pages in use to the pool's beginning: (pages moved, in use, first number past them).  The host waits."""
        n = B.fcp_cache_scratch_bytes(B.FCP_SCRATCH_CACHE_COMPACT, self.cache, *self.pages.shape)
        B.fcp_cache_compact(self.cache, self.pages, self.kv_len, self.pages, self.counts, torch.empty(n, dtype=torch.uint8, device=self.device))
        return tuple(self.counts.tolist())

    def sequences(self):
        """[n_prompts, beams, selections] int64: the tokens of every beam, from the choices and whom they continue; -1 where a beam had no candidate.  The host waits."""
        out = np.full((self.n, self.beams, len(self.history)), -1, np.int64)
        row = np.arange(self.n * self.beams)
        for t in range(len(self.history) - 1, -1, -1):
            parent, token = (x.cpu().numpy().reshape(-1) for x in self.history[t])
            out.reshape(-1, len(self.history))[:, t] = np.where(row >= 0, token[row], -1)
            row = np.where(row >= 0, parent[row], -1)
        return out


def main():
    g = torch.Generator(device="cuda").manual_seed(0)
    lens, hq, hkv, D = [700, 150, 33, 1200], 32, 8, 128
    turns, magnitude = B.fcp_rotary_frequencies(D, 500000.0, B.FCP_ROTARY_PARTS, factor=4.0, original_len=8192)
    dec = CacheDecoder(len(lens), 256, 64, hq, hkv, D, turns=turns, magnitude=magnitude)
    rows = lambda n, h: torch.randn(n, h, D, generator=g, device="cuda").to(torch.bfloat16)
    o, _ = dec.prefill(rows(sum(lens), hq), rows(sum(lens), hkv), rows(sum(lens), hkv), lens)
    print("prompts of", lens, "tokens:", tuple(o.shape), "rows, pages in use:", int((dec.pages >= 0).sum()))
    for t in range(8):
        o, lse = dec.step(rows(len(lens), hq), rows(len(lens), hkv), rows(len(lens), hkv), [1] * len(lens))
    print("8 tokens each: cached", dec.kv_len.tolist(), "mean LSE %.3f" % float(lse.mean()))
    kept = dec.evict(512, n_first=4, n_recent=64)
    print("cut to 512: cached", dec.kv_len.tolist(), "head 0 of sequence 0 keeps", kept[0, 0, :8].tolist(), "...; pages in use:", int((dec.pages >= 0).sum()))
    o, lse = dec.step(rows(9, hq), rows(9, hkv), rows(9, hkv), [1, 5, 0, 3])
    print("1, 5, 0 and 3 tokens more: cached", dec.kv_len.tolist(), "mean LSE %.3f" % float(lse.mean()))
    beams = BeamDecoder(len(lens), 4, 256, 64, hq, hkv, D, turns=turns, magnitude=magnitude)
    beams.prefill(rows(sum(lens), hq), rows(sum(lens), hkv), rows(sum(lens), hkv), lens)
    for t in range(8):
        beams.select(3 * torch.randn(len(lens) * (4 if t else 1), 32000, generator=g, device="cuda"))
        o, lse = beams.step(rows(4 * len(lens), hq), rows(4 * len(lens), hkv), rows(4 * len(lens), hkv))
    print("4 beams each, 8 tokens: the best of the first prompt", beams.sequences()[0, 0].tolist(), "at %.2f;" % float(beams.score[0]), "pages moved, in use, end:", beams.compact())


if __name__ == "__main__":
    main()
