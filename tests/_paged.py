"""Random batches over a paged cache and the operators' definitions in 64 bits (numpy only)."""
import numpy as np

HALF_STEP = {"float16": 2.0 ** -11, "bfloat16": 2.0 ** -8, "float32": 2.0 ** -24}     # largest relative rounding error


def to_bf16(x):
    """Rounded to bfloat16 (ties to even), kept in float32."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)


def rounded(x, dtype):
    return x.astype(np.float16).astype(np.float32) if dtype == "float16" else to_bf16(x) if dtype == "bfloat16" else x.astype(np.float32)


class Batch:
    """Sequences with ctx[s] cached positions and nodes[s] rows; pages in a shuffled order, spare ones behind them."""

    def __init__(self, seed, ctx, nodes, page, layers=1, kv_heads=2, q_heads=4, dim=64, dtype="float16", pad=0, spare=2):
        rs = self.rs = np.random.RandomState(seed)
        self.ctx, self.nodes = np.array(ctx, np.int32), np.array(nodes, np.int32)
        self.page, self.layers, self.kv_heads, self.q_heads, self.dim, self.dtype = page, layers, kv_heads, q_heads, dim, dtype
        self.row_begin = np.concatenate([[0], np.cumsum(self.nodes)]).astype(np.int32)
        self.live = int(self.row_begin[-1])
        self.n_tok = self.live + pad
        used = -(-(self.ctx + self.nodes) // page)
        self.n_pages = int(used.sum()) + spare
        ids = rs.permutation(self.n_pages)
        self.table = np.full((len(ctx), max(1, int(used.max())) + 1), -1, np.int32)
        at = 0
        for s, u in enumerate(used):
            self.table[s, :u] = ids[at:at + u]
            at += u
        shape = (layers, self.n_pages, kv_heads, page, dim)
        self.k = rounded(rs.standard_normal(shape).astype(np.float32), dtype)
        self.v = rounded(rs.standard_normal(shape).astype(np.float32), dtype)

    def place(self, s, slot):
        return int(self.table[s, slot // self.page]), slot % self.page

    def entries(self, a, s, layer, n):
        """[n][kv_heads][dim] of sequence s."""
        return np.stack([a[layer, self.table[s, j // self.page], :, j % self.page] for j in range(n)]) if n else np.zeros((0, self.kv_heads, self.dim))

    def trees(self, words=1, chain=False):
        """Random trees as bits of ancestors-and-self, [n_tok][words] int64, and their depths."""
        mask, depth = np.zeros((self.n_tok, words), np.uint64), np.zeros(self.n_tok, np.int32)
        for s, n in enumerate(self.nodes):
            b = self.row_begin[s]
            for i in range(n):
                parent = (i - 1 if chain else int(self.rs.randint(max(0, i - 5), i))) if i else -1
                if parent >= 0:
                    mask[b + i] = mask[b + parent]
                    depth[b + i] = depth[b + parent] + 1
                if i < 64 * words:
                    mask[b + i, i // 64] |= np.uint64(1 << (i % 64))
        return mask.view(np.int64), depth

    def sees(self, s, mask):
        """[rows][slots] of sequence s."""
        c, n, b = int(self.ctx[s]), int(self.nodes[s]), int(self.row_begin[s])
        out = np.ones((n, c + n), bool)
        for i in range(n):
            if mask is None:
                out[i, c:] = np.arange(n) <= i
            else:
                w = mask[b + i].view(np.uint64)
                out[i, c:] = [a < 64 * len(w) and bool(int(w[a // 64]) >> (a % 64) & 1) for a in range(n)]
        return out


def attention(batch, layer, q, mask, scale):
    """(out, lse, bound on |out error| apart from the final rounding) in 64 bits, rows of padding left NaN."""
    group = batch.q_heads // batch.kv_heads
    u = HALF_STEP[batch.dtype]
    out = np.full((batch.n_tok, batch.q_heads, batch.dim), np.nan)
    lse = np.full((batch.n_tok, batch.q_heads), np.nan)
    bound, lse_bound = np.zeros_like(out), np.zeros_like(lse)
    for s in range(len(batch.ctx)):
        n = int(batch.ctx[s] + batch.nodes[s])
        k, v = (batch.entries(a, s, layer, n).astype(np.float64) for a in (batch.k, batch.v))
        see = batch.sees(s, mask)
        for i in range(int(batch.nodes[s])):
            t = int(batch.row_begin[s]) + i
            for h in range(batch.q_heads):
                g = h // group
                at = np.flatnonzero(see[i])
                if at.size == 0:
                    out[t, h], lse[t, h] = 0.0, -np.inf
                    continue
                qq = q[t, h].astype(np.float64)
                kk, vv = k[at, g], v[at, g]
                x = scale * (kk @ qq)
                top = x.max()
                p = np.exp(x - top)
                total = p.sum()
                out[t, h], lse[t, h] = (p / total) @ vv, top + np.log(total)
                # a score: dim + 2 roundings of 2^-24 relative to the sum of magnitudes; a probability: the error of its score
                # and of the reference, an ex2 of 2^-21, its rounding to the cache's type; the sums: 2^-24 per addition of a row
                d_score = (batch.dim + 4) * 2.0 ** -24 * scale * (np.abs(kk) @ np.abs(qq)).max() + np.abs(x).max() * 2.0 ** -22
                rel = u + 2 * d_score + 2.0 ** -20 + at.size * 2.0 ** -24
                bound[t, h] = (p / total) @ np.abs(vv) * rel + np.abs(out[t, h]) * rel
                lse_bound[t, h] = 2 * d_score + 2.0 ** -20 + at.size * 2.0 ** -24 + np.abs(lse[t, h]) * 2.0 ** -22
    return out, lse, bound, lse_bound


def rotate(x, pos, theta, mode):
    """[n][heads][dim] turned in 64 bits."""
    dim = x.shape[-1]
    angle = pos.astype(np.float64)[:, None] * np.power(np.float64(np.float32(theta)), -2.0 * np.arange(dim // 2) / dim)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    x = x.astype(np.float64)
    out = np.empty_like(x)
    if mode == 0:
        a, b = x[..., :dim // 2], x[..., dim // 2:]
        out[..., :dim // 2], out[..., dim // 2:] = a * c - b * s, a * s + b * c
    else:
        a, b = x[..., 0::2], x[..., 1::2]
        out[..., 0::2], out[..., 1::2] = a * c - b * s, a * s + b * c
    return out


def beam_select(logits, cum, keep, finished=None, end=0):
    """Scores (64 bits), parents and tokens of the best candidates, per request."""
    n_req, n_beams, vocab = logits.shape
    score = np.full((n_req, keep), -np.inf)
    parent, token = np.zeros((n_req, keep), np.int32), np.full((n_req, keep), -1, np.int32)
    for r in range(n_req):
        cand = []
        for b in range(n_beams):
            c = np.float64(cum[r, b])
            if not c > -np.inf:
                continue
            if finished is not None and finished[r, b]:
                cand.append(np.array([[c], [b * vocab + end]]))
                continue
            x = logits[r, b].astype(np.float64)
            x = np.where(np.isnan(x), -np.inf, np.minimum(x, np.finfo(np.float32).max))
            top = x.max()
            if top == -np.inf:
                continue
            at = np.flatnonzero(x > -np.inf)
            cand.append(np.stack([c + ((x[at] - top) - np.log(np.exp(x[at] - top).sum())), b * vocab + at.astype(np.float64)]))
        if not cand:
            continue
        cand = np.concatenate(cand, 1)
        order = np.lexsort((cand[1], -cand[0]))[:keep]
        score[r, :order.size] = cand[0, order]
        flat = cand[1, order].astype(np.int64)
        parent[r, :order.size], token[r, :order.size] = flat // vocab, flat % vocab
    return score, parent, token
