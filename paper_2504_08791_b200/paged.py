"""Page tables on the host, and the two loops that need caches whose sequences fork: speculative decoding with a drafted
TREE of tokens (paper Appendix A.9 and A.12 verify a chain) and beam search.

A ``PageTable`` hands out pages of a ``binding.PagedCache`` and counts who uses them; ``PagedStepper`` runs model steps
over it (``prima_embed`` / ``prima_forward_window_paged`` per window / ``prima_logits``).  Only orchestration lives here;
torch is used for the device buffers.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Callable, List, Optional, Sequence, Tuple

import numpy as np

from .speculative import SpeculativeStats


class PageTable:
    """Pages 0 .. n_pages - 1, each with the number of sequences that use it."""

    def __init__(self, n_pages: int, page_size: int):
        self.page_size = page_size
        self.users = [0] * n_pages
        self.free = list(range(n_pages - 1, -1, -1))

    def take(self) -> int:
        if not self.free:
            raise RuntimeError("the paged cache is full")
        page = self.free.pop()
        self.users[page] = 1
        return page

    def share(self, page: int) -> int:
        self.users[page] += 1
        return page

    def drop(self, page: int):
        self.users[page] -= 1
        if self.users[page] == 0:
            self.free.append(page)

    def grow(self, pages: List[int], n_positions: int):
        """Appends pages of its own to a sequence's list until it holds n_positions."""
        while len(pages) * self.page_size < n_positions:
            pages.append(self.take())

    def reorder(self, rows: List[List[int]], lengths: Sequence[int], parents: Sequence[int], fresh: Sequence[int]) -> List[List[int]]:
        """What ``PagedCache.reorder`` does to the tables, on the host: the new rows.  A page of ``fresh`` that is not
        needed goes back."""
        seen, new = set(), []
        for r, p in enumerate(parents):
            used = -(-lengths[p] // self.page_size)
            pages = rows[p][:used]
            if lengths[p] % self.page_size and p in seen:
                row = [self.share(x) for x in pages[:-1]] + [fresh[r]]
            else:
                row = [self.share(x) for x in pages]
                self.drop(fresh[r])
            seen.add(p)
            new.append(row)
        for row in rows:
            for x in row:
                self.drop(x)
        return new


class PagedStepper:
    """One model behind a context, its sequences in a paged cache."""

    def __init__(self, ctx, k_pages, v_pages, windows: Optional[Sequence[int]] = None):
        import torch
        from . import binding
        cfg = ctx.cfg
        self.binding, self.torch, self.ctx, self.cfg = binding, torch, ctx, cfg
        self.pool = binding.PagedCache(k_pages, v_pages, rope_theta=cfg["rope_theta"], rope_mode=cfg.get("rope_mode", 0))
        self.pages = PageTable(self.pool.n_pages, self.pool.page_size)
        bounds = list(windows) if windows is not None else [0, cfg["n_layers"]]
        if bounds[0] != 0 or bounds[-1] != cfg["n_layers"] or any(b <= a for a, b in zip(bounds, bounds[1:])):
            raise ValueError("windows must be ascending layer boundaries from 0 to n_layers")
        self.bounds, self.max_n_tok = bounds, cfg.get("max_n_tok", binding.MAX_N_TOK)
        self.hid = torch.empty((self.max_n_tok, cfg["hidden"]), dtype=torch.float32, device=k_pages.device)
        self.logits = torch.empty((self.max_n_tok, cfg["vocab"]), dtype=torch.float32, device=k_pages.device)

    def on_stream(self):
        """torch's current stream becomes the context's: the small arrays of a step are then uploaded, and their memory is
        used again, in the order of the steps that read them."""
        return self.torch.cuda.stream(self.ctx._stream)

    def _gpu(self, a, dtype=np.int32):
        with self.on_stream():
            return self.torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to(self.hid.device)

    def table_of(self, rows: Sequence[Sequence[int]]):
        width = max(1, max(len(r) for r in rows))
        return self._gpu([list(r) + [-1] * (width - len(r)) for r in rows])

    def batch(self, rows: Sequence[Sequence[int]], lengths: Sequence[int], counts: Sequence[int], pos=None, mask=None):
        """A step of counts[s] tokens of sequence s, whose pages are rows[s] and which holds lengths[s] positions."""
        begin = np.concatenate([[0], np.cumsum(counts)])
        return self.binding.PagedBatch(self.table_of(rows), self._gpu(begin), self._gpu(lengths), int(begin[-1]), pos=None if pos is None else self._gpu(pos),
                                       mask=None if mask is None else self._gpu(mask, np.int64))

    def step(self, tokens: Sequence[int], batch):
        """Runs the tokens; their logits stay in ``self.logits[:n]``."""
        n = len(tokens)
        if not 1 <= n <= self.max_n_tok or n != batch.n_tok:
            raise ValueError("between 1 and max_n_tok tokens per step, as many as the batch has rows")
        hid = self.hid[:n]
        self.ctx.embed(list(tokens), hid)
        for lb, le in zip(self.bounds, self.bounds[1:]):
            self.ctx.forward_window_paged(self.pool, lb, le, hid, hid, batch)
        self.ctx.logits(hid, n, self.logits[:n])
        return self.logits[:n]

    def prefill(self, tokens: Sequence[int], pages: List[int], length: int = 0) -> int:
        """Reads a prompt into the sequence with these pages; returns its new length."""
        for at in range(0, len(tokens), self.max_n_tok):
            part = tokens[at:at + self.max_n_tok]
            self.pages.grow(pages, length + len(part))
            self.step(part, self.batch([pages], [length], [len(part)]))
            length += len(part)
        return length


# ---- trees of drafted tokens --------------------------------------------------------------------------------------
@dataclass
class DraftTree:
    """Node 0 is the newest token (in no cache yet); parents come before their children."""
    tokens: List[int]
    parents: List[int]

    def depths(self) -> List[int]:
        out: List[int] = []
        for p in self.parents:
            out.append(0 if p < 0 else out[p] + 1)
        return out

    def mask(self) -> np.ndarray:
        """[nodes, words] int64: bit a of row i, node a is i or an ancestor of i."""
        n = len(self.tokens)
        words = -(-n // 64)
        m = np.zeros((n, words), np.uint64)
        for i, p in enumerate(self.parents):
            if not -1 <= p < i or (p < 0) != (i == 0):
                raise ValueError("a tree has one root, node 0, and parents come before their children")
            if p >= 0:
                m[i] = m[p]
            m[i, i // 64] |= np.uint64(1 << (i % 64))
        return m.view(np.int64)

    def accept(self, choices: Sequence[int]) -> Tuple[List[int], int]:
        """choices[i]: the target's own next token after node i.  The nodes of the accepted path (from node 0 down, as
        long as a child is what the target chose) and the target's token after its end."""
        path = [0]
        while True:
            want = int(choices[path[-1]])
            child = next((i for i in range(path[-1] + 1, len(self.tokens)) if self.parents[i] == path[-1] and self.tokens[i] == want), None)
            if child is None:
                return path, want
            path.append(child)


class TreeSpeculativeDecoder:
    """Greedy speculative decoding whose drafts are trees: ``propose(history, limit)`` returns the drafted tree behind
    the newest token (at most ``limit`` nodes, node 0 the newest token itself), the target runs ONE step over all of its
    nodes, the path that agrees with the target's own choices is kept and moved into place (``PagedCache.accept``).
    Whatever is proposed, the output is what greedy decoding with the target alone gives."""

    def __init__(self, target: PagedStepper, propose: Callable[[List[int], int], DraftTree]):
        self.target, self.propose = target, propose

    def generate(self, history: Sequence[int], pages: List[int], length: int, n_new: int):
        """``history``: all tokens so far; the last of them is not in the cache, the ``length`` before it are, on
        ``pages`` (extended here).  Returns the n_new tokens that follow and the statistics of the run."""
        t = self.target
        history, out, stats = [int(x) for x in history], [], SpeculativeStats()
        while len(out) < n_new:
            tree = self.propose(history, t.max_n_tok)
            if not tree.tokens or tree.tokens[0] != history[-1] or len(tree.tokens) > t.max_n_tok:
                raise ValueError("a draft begins with the newest token and fits one step of the target")
            n = len(tree.tokens)
            t.pages.grow(pages, length + n)
            pos = [length + d for d in tree.depths()]
            batch = t.batch([pages], [length], [n], pos=pos, mask=tree.mask())
            choices = t.ctx.argmax(t.step(tree.tokens, batch), n)
            path, bonus = tree.accept(choices)
            t.pool.accept(batch, t._gpu([path]), t._gpu([len(path)]), stream=t.ctx._stream)
            new = [tree.tokens[i] for i in path[1:]] + [bonus]
            length += len(path)
            history += new
            out += new
            stats.cycles += 1
            stats.proposed += n - 1
            stats.accepted += len(path) - 1
            stats.per_cycle.append(len(new))
        return out[:n_new], stats


# ---- beam search ----------------------------------------------------------------------------------------------------
class BeamDecoder:
    """Beam search of one request: every step runs one token of each beam (``prima_forward_window_paged``), chooses the
    best continuations (``prima_beam_select``) and reorders the page tables (``prima_paged_reorder``)."""

    def __init__(self, model: PagedStepper, n_beams: int, end_token: Optional[int] = None):
        if not 1 <= n_beams <= model.max_n_tok:
            raise ValueError("one token of every beam must fit one step")
        self.model, self.n_beams, self.end_token = model, n_beams, end_token

    def generate(self, prompt: Sequence[int], n_new: int) -> List[Tuple[float, List[int]]]:
        """(sum of log probabilities, tokens) of the beams after n_new steps (fewer where a beam has ended), best first."""
        rows, fresh = [[]], []
        try:
            with self.model.on_stream():
                return self._generate(prompt, n_new, rows, fresh)
        finally:      # a full cache too leaves no page behind
            for pages in (*rows, fresh):
                for p in pages:
                    self.model.pages.drop(p)

    def _generate(self, prompt: Sequence[int], n_new: int, rows: List[List[int]], fresh: List[int]):
        m, torch, n = self.model, self.model.torch, self.n_beams
        dev = m.hid.device
        length = m.prefill(prompt[:-1], rows[0]) if len(prompt) > 1 else 0
        rows += [[m.pages.share(p) for p in rows[0]] for _ in range(n - 1)]
        # all beams start as the prompt, but only the first one counts; their last pages become their own as they grow
        lengths, tokens = [length] * n, [[] for _ in range(n)]
        feed = [int(prompt[-1])] * n
        score = torch.full((1, n), -float("inf"), device=dev)
        score[0, 0] = 0.0
        done = np.zeros(n, bool)
        parent, token = (torch.zeros((1, n), dtype=torch.int32, device=dev) for _ in range(2))
        for step in range(n_new):
            alive = [0] if step == 0 else list(range(n))
            for b in alive:
                m.pages.grow(rows[b], lengths[b] + 1)
            logits = m.step([feed[b] for b in alive], m.batch([rows[b] for b in alive], [lengths[b] for b in alive], [1] * len(alive)))
            if step == 0:
                logits = logits.expand(n, -1)
                lengths[0] += 1
            else:
                lengths = [x + 1 for x in lengths]
            new_score = torch.empty_like(score)
            m.binding.prima_beam_select(logits.contiguous()[None], score, new_score, parent, token, finished=m._gpu([done], np.uint8) if done.any() else None,
                                        end_token=self.end_token if done.any() else -1)
            while len(fresh) < n:
                fresh.append(m.pages.take())
            table = m.table_of(rows)
            out = torch.empty_like(table), torch.empty(n, dtype=torch.int32, device=dev)
            m.pool.reorder(table, m._gpu(lengths), parent, m._gpu(fresh), *out)
            parents, words = parent[0].tolist(), token[0].tolist()
            rows[:] = m.pages.reorder(rows, lengths, parents, fresh)
            fresh.clear()
            lengths = [lengths[p] for p in parents]
            ended = [bool(done[p]) for p in parents]
            tokens = [tokens[p] + ([] if e else [w]) for p, w, e in zip(parents, words, ended)]
            done = np.array([e or (self.end_token is not None and w == self.end_token) for e, w in zip(ended, words)])
            feed, score = [max(0, w) for w in words], new_score
            if done.all():
                break
        return list(zip(score[0].tolist(), tokens))
