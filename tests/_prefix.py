"""Batches behind shared prefixes, and 64-bit definitions of the operators of long prompts and bounded caches (numpy only)."""
import numpy as np

from tests import _paged
from tests._paged import HALF_STEP, Batch


class PrefixBatch(Batch):
    """A batch whose sequences groups[p] .. groups[p + 1] - 1 share a prefix of prefix[p] positions, on pages of its own."""

    def __init__(self, seed, ctx, nodes, prefix, groups, page, **kw):
        pages = [-(-n // page) for n in prefix]
        super().__init__(seed, ctx, nodes, page, spare=sum(pages) + 2, **kw)
        used = set(self.table[self.table >= 0].tolist())
        free = self.rs.permutation([i for i in range(self.n_pages) if i not in used])
        self.prefix, self.groups = np.array(prefix, np.int32), np.array(groups, np.int32)
        self.prefix_table = np.full((len(prefix), max(1, max(pages)) + 1), -1, np.int32)
        at = 0
        for p, n in enumerate(pages):
            self.prefix_table[p, :n] = free[at:at + n]
            at += n

    def prefix_of(self, s):
        for p in range(len(self.prefix)):
            if self.groups[p] <= s < self.groups[p + 1]:
                return p
        return None

    def prefix_entries(self, a, p, layer):
        n = int(self.prefix[p]) if p is not None else 0
        if not n:
            return np.zeros((0, self.kv_heads, self.dim))
        return np.stack([a[layer, self.prefix_table[p, j // self.page], :, j % self.page] for j in range(n)])


def score_bound(q, k, x, scale):
    """Largest error of a score in 32 bits: dim + 4 roundings of 2^-24 of the sum of magnitudes, and two of the score itself."""
    return (q.shape[-1] + 4) * 2.0 ** -24 * scale * (np.abs(k) @ np.abs(q)).max() + np.abs(x).max() * 2.0 ** -22


def prefix_attention(b, layer, q, mask, scale):
    """(out, lse, bound on |out error| apart from the final rounding, bound of lse), rows of padding left NaN."""
    group, u = b.q_heads // b.kv_heads, HALF_STEP[b.dtype]
    out, lse = np.full((b.n_tok, b.q_heads, b.dim), np.nan), np.full((b.n_tok, b.q_heads), np.nan)
    bound, lse_bound = np.zeros_like(out), np.zeros_like(lse)
    entries = {p: [b.prefix_entries(a, p, layer).astype(np.float64) for a in (b.k, b.v)] for p in [None, *range(len(b.prefix))]}
    for s in range(len(b.ctx)):
        n = int(b.ctx[s] + b.nodes[s])
        shared = entries[b.prefix_of(s)]
        k, v = (np.concatenate([f, b.entries(a, s, layer, n).astype(np.float64)]) for f, a in zip(shared, (b.k, b.v)))
        see = np.concatenate([np.ones((int(b.nodes[s]), len(shared[0])), bool), b.sees(s, mask)], 1)
        for i in range(int(b.nodes[s])):
            t, at = int(b.row_begin[s]) + i, np.flatnonzero(see[i])
            for h in range(b.q_heads):
                if at.size == 0:
                    out[t, h], lse[t, h] = 0.0, -np.inf
                    continue
                qq, kk, vv = q[t, h].astype(np.float64), k[at, h // group], v[at, h // group]
                x = scale * (kk @ qq)
                top = x.max()
                p = np.exp(x - top)
                total = p.sum()
                out[t, h], lse[t, h] = (p / total) @ vv, top + np.log(total)
                # as for trees: a probability has the error of its score and of the reference, an ex2 of 2^-21 and its rounding
                # to the cache's type; the sums 2^-24 for each addition of a row
                d = score_bound(qq, kk, x, scale)
                rel = u + 2 * d + 2.0 ** -20 + at.size * 2.0 ** -24
                bound[t, h] = (p / total) @ np.abs(vv) * rel + np.abs(out[t, h]) * rel
                lse_bound[t, h] = 2 * d + 2.0 ** -20 + at.size * 2.0 ** -24 + np.abs(lse[t, h]) * 2.0 ** -22
    return out, lse, bound, lse_bound


def weights(b, layer, q, lse, mask, scale, weight_in, decay):
    """(what every slot has after the step, bound on its error), [sequences][KV heads][slots up to the longest]."""
    group = b.q_heads // b.kv_heads
    longest = int((b.ctx + b.nodes).max())
    out, bound = np.zeros((len(b.ctx), b.kv_heads, longest)), np.zeros((len(b.ctx), b.kv_heads, longest))
    for s in range(len(b.ctx)):
        c, n, first = int(b.ctx[s]), int(b.nodes[s]), int(b.row_begin[s])
        if not n:
            continue
        k, see = b.entries(b.k, s, layer, c + n).astype(np.float64), b.sees(s, mask)
        for h in range(b.q_heads):
            g = h // group
            for i in range(n):
                z = np.float64(lse[first + i, h])
                if z == -np.inf:
                    continue
                qq = q[first + i, h].astype(np.float64)
                x = scale * (k[:, g] @ qq)
                p = np.where(see[i], np.exp(x - z), 0.0)
                # the score's error, that of lse times log2(e) and of their difference (three roundings of both), an ex2 of 2^-21
                rel = (b.dim + 4) * 2.0 ** -24 * scale * (np.abs(k[:, g]) @ np.abs(qq)) + (np.abs(x) + abs(z)) * 3 * 2.0 ** -24 + 2.0 ** -21
                out[s, g, :c + n] += p
                bound[s, g, :c + n] += p * rel
        # sums of `rows` terms in 32 bits, in any order
        bound[s] += out[s] * (n * group + 2) * 2.0 ** -24
        if weight_in is not None:
            had = decay * weight_in[s, :, :c].astype(np.float64)
            out[s, :, :c] += had
            bound[s, :, :c] += (np.abs(had) + np.abs(out[s, :, :c])) * 2.0 ** -23
    return out, bound


def choose(weight, born, n, keep, first, recent_from):
    """Slots kept of the n of one KV head, ascending, and the slot whose entry each of the first m slots holds afterwards."""
    m = min(n, keep)
    w = weight[:n].astype(np.float64)
    w = np.where(np.isnan(w), -np.inf, w)
    rank = np.isnan(weight[:n]).astype(int)      # NaN behind -infinity
    stays = born[:n] < first
    if recent_from is not None:
        stays |= born[:n] >= recent_from
    w, rank = np.where(stays, 0.0, w), np.where(stays, 0, rank)      # protected entries are equal
    order = np.lexsort((np.arange(n), -w, rank, ~stays))
    w_kept = np.sort(order[:m])
    source = np.arange(m)
    holes = np.setdiff1d(source, w_kept)
    source[holes] = w_kept[w_kept >= m]
    return w_kept, source


def norm_and_turn(x, gain, eps, angle, mode):
    """[n][heads][dim] normed (gain [heads][dim] or None) and turned by angle [n][dim / 2], in 64 bits."""
    y = x.astype(np.float64)
    if gain is not None:
        y = gain * y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps)
    half = y.shape[-1] // 2
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    out = np.empty_like(y)
    lo, hi = (slice(0, half), slice(half, None)) if mode == 0 else (slice(0, None, 2), slice(1, None, 2))
    out[..., lo], out[..., hi] = y[..., lo] * c - y[..., hi] * s, y[..., lo] * s + y[..., hi] * c
    return out, y
