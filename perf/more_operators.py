"""The operators of long prompts and bounded caches over a paged cache, as cases to be measured.

  norm     RMS norm of every query and key head, rotation by positions on several axes, keys and values appended
  prefix   attention of a batch whose sequences share long prefixes, each prefix read once for all that share it
  weights  the attention weight that every cached position received in a step, added to what it had
  evict    the entries of largest weight kept, moved together into the first slots of the cache

``run`` computes each in plain torch operations, or, where ``own`` is true, by the package's entry points.
Cache layout: [layers][pages][KV heads][page size][head size]; sequence s holds position j in page
table[s][j // page size] at row j % page size.  Lengths follow from the case alone, values from the seed.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_THETA = 1e6
_EPS = 1e-6

# Which axis turns pair i of a head of 128 or 64, by the kind of the case.
#   text       one axis
#   sections   time, height and width own a stretch of pairs each (16 + 24 + 24 of 64)
#   turns      pairs take the three axes in turn, the slowest quarter follows time
#   grid       two axes for image patches, frequencies counted anew on each; the last quarter is not turned


def _axes(kind, dim):
    """(axis of every pair, -1: not turned; number of the frequency of every pair; axes)"""
    half = dim // 2
    i = np.arange(half)
    if kind == "text":
        return np.zeros(half, int), i, 1
    if kind == "sections":
        return np.where(i < half // 4, 0, np.where(i < half // 4 + 3 * half // 8, 1, 2)), i, 3
    if kind == "turns":
        return np.where(i < 3 * half // 4, i % 3, 0), i, 3
    quarter = half // 4
    return np.where(i < 3 * quarter // 2, 0, np.where(i < 3 * quarter, 1, -1)), 2 * (i % (3 * quarter // 2)), 2


def _cases():
    return [
        # one token of one request, 8B-shaped heads: what a decoding step pays per layer
        {"name": "norm_one", "op": "norm", "dtype": "f16", "src": "f32", "seqs": 1, "nodes": [1, 1], "ctx": [1024, 1024],
         "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "mode": 0, "axes": "text", "head_gain": False, "pad": 0},
        # drafted tokens of a batch of requests, heads of 64 with a gain for each, neighbouring pairs, axes in turn, padded rows
        {"name": "norm_drafts", "op": "norm", "dtype": "f16", "src": "f16", "seqs": 48, "nodes": [1, 7], "ctx": [17, 4000],
         "q_heads": 24, "kv_heads": 4, "dim": 64, "page": 32, "mode": 1, "axes": "turns", "head_gain": True, "pad": 3},
        # prompts of text and images of five requests, 32B-shaped heads
        {"name": "norm_prompts", "op": "norm", "dtype": "bf16", "src": "bf16", "seqs": 5, "nodes": [900, 4001], "ctx": [0, 0],
         "q_heads": 40, "kv_heads": 8, "dim": 128, "page": 64, "mode": 0, "axes": "sections", "head_gain": False, "pad": 0},
        # four beams over their prompt, 8B-shaped: the smallest batch that shares anything
        {"name": "prefix_beams", "op": "prefix", "dtype": "f16", "prefixes": 1, "prefix": [1000, 1000], "seqs": 4, "nodes": [1, 1], "ctx": [3, 20],
         "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "pad": 0},
        # requests of three system prompts, heads of 64, short drafts, padded rows
        {"name": "prefix_three", "op": "prefix", "dtype": "f16", "prefixes": 3, "prefix": [300, 6001], "seqs": 45, "nodes": [1, 5], "ctx": [1, 900],
         "q_heads": 32, "kv_heads": 8, "dim": 64, "page": 32, "pad": 3},
        # a batch behind one long system prompt, 32B-shaped heads (five query heads share a KV head)
        {"name": "prefix_batch", "op": "prefix", "dtype": "bf16", "prefixes": 1, "prefix": [8192, 8192], "seqs": 64, "nodes": [1, 1], "ctx": [1, 1500],
         "q_heads": 40, "kv_heads": 8, "dim": 128, "page": 64, "pad": 0},
        # many requests over one long document, 70B-shaped heads
        {"name": "prefix_document", "op": "prefix", "dtype": "f16", "prefixes": 1, "prefix": [32765, 32765], "seqs": 192, "nodes": [1, 1], "ctx": [10, 600],
         "q_heads": 64, "kv_heads": 8, "dim": 128, "page": 64, "pad": 0},
        # one token of one request, 8B-shaped heads, per layer of a decoding step
        {"name": "weights_one", "op": "weights", "dtype": "f16", "seqs": 1, "nodes": [1, 1], "ctx": [4000, 4000],
         "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "decay": 1.0, "first_time": False},
        # single tokens of a batch of requests, 32B-shaped heads, older weight counting less
        {"name": "weights_batch", "op": "weights", "dtype": "bf16", "seqs": 48, "nodes": [1, 1], "ctx": [1, 8192],
         "q_heads": 40, "kv_heads": 8, "dim": 128, "page": 32, "decay": 0.98, "first_time": False},
        # the last 64 rows of a prompt of 32,768 tokens say which of its entries stay, 70B-shaped heads
        {"name": "weights_prompt", "op": "weights", "dtype": "f16", "seqs": 1, "nodes": [64, 64], "ctx": [32704, 32704],
         "q_heads": 64, "kv_heads": 8, "dim": 128, "page": 64, "decay": 1.0, "first_time": True},
        # a request's cache brought back to 2048 entries after 250 tokens, all 32 layers of an 8B-shaped model
        {"name": "evict_one", "op": "evict", "dtype": "f16", "seqs": 1, "ctx": [2298, 2298], "keep": [2048, 2048], "kv_heads": 8, "dim": 128,
         "page": 16, "layers": 32, "first": 4, "recent": 256},
        # prompts of six requests cut to about a thousand entries each, some shorter than that
        {"name": "evict_prompts", "op": "evict", "dtype": "bf16", "seqs": 6, "ctx": [700, 16001], "keep": [1000, 1100], "kv_heads": 8, "dim": 128,
         "page": 64, "layers": 10, "first": 4, "recent": 64},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def span(lo, hi):
        a, b = log(lo, hi), log(lo, hi)
        return [min(a, b), max(a, b)]

    op = rng.choice(["norm", "prefix", "prefix", "weights", "weights", "evict"])
    case = {"op": op, "dtype": rng.choice(["f16", "bf16"]), "dim": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128]),
            "kv_heads": rng.choice([1, 2, 4, 8])}
    group = rng.choice([1, 2, 3, 4, 5, 7, 8])
    if op == "norm":
        seqs = log(1, 64)
        case |= {"src": rng.choice(["f32", case["dtype"]]), "seqs": seqs, "nodes": span(1, max(1, 6000 // seqs)), "ctx": span(1, 4096),
                 "mode": rng.choice([0, 1]), "axes": rng.choice(["text", "sections", "turns", "grid"]), "head_gain": rng.random() < 0.5,
                 "pad": rng.choice([0, 0, 5])}
    elif op == "prefix":
        prefixes = rng.choice([1, 1, 1, 2, 3])
        seqs = log(2 * prefixes, 192)
        case |= {"prefixes": prefixes, "prefix": span(64, 32768 // prefixes), "seqs": seqs, "nodes": span(1, max(1, min(8, 192 // seqs))),
                 "ctx": span(1, min(2000, 60000 // seqs)), "pad": rng.choice([0, 0, 3])}
    elif op == "weights":
        few = rng.random() < 0.6
        seqs = log(1, 48) if few else 1
        case |= {"seqs": seqs, "nodes": [1, 1] if few else span(2, 64), "ctx": span(1, 8192 if few else 32000), "decay": rng.choice([1.0, 0.98, 0.5]),
                 "first_time": rng.random() < 0.3}
    else:
        seqs, layers = log(1, 6), log(1, 32)
        case |= {"seqs": seqs, "ctx": span(20, max(40, 90000 // (seqs * layers))), "layers": layers, "first": rng.choice([0, 4]), "recent": log(1, 64)}
        case["keep"] = span(10, case["ctx"][1])
    if op != "evict":
        case["q_heads"] = group * case["kv_heads"]
    return _plain_values(case)


def _plain_values(case):
    """A case holds numbers, texts and truth values: a span becomes two numbers."""
    out = {}
    for k, v in case.items():
        if isinstance(v, list):
            out[k + "_min"], out[k + "_max"] = v
        else:
            out[k] = v
    return out


def listed():
    return [_plain_values(c) for c in _cases()]


def _spread(case, key, n):
    """n lengths between the case's two bounds, even over their logarithm, in a mixed order; the first is the largest."""
    lo, hi = case[key + "_min"], case[key + "_max"]
    at = np.modf(np.arange(n) * 0.6180339887498949)[0]
    return np.rint(np.exp(np.log(hi + 1) + (np.log(lo + 1) - np.log(hi + 1)) * at) - 1).astype(np.int64).clip(lo, hi)


def _lengths(case):
    """(positions in front of the step, rows of the step) of every sequence."""
    return _spread(case, "ctx", case["seqs"]), _spread(case, "nodes", case["seqs"])[::-1].copy()


def _groups(case):
    """First sequence of every prefix, and the end: unequal shares."""
    n, p = case["seqs"], case["prefixes"]
    at = np.sort(np.array([n * (i + 0.35 * (i % 2)) / p for i in range(p)]).astype(int))
    return np.concatenate([at, [n]]).astype(np.int32)


def _pages_of(case, lengths):
    return -(-lengths // case["page"])


def _cache(case, n_pages, gen):
    shape = (case.get("layers", 1), n_pages, case["kv_heads"], case["page"], case["dim"])
    return [torch.randn(shape, generator=gen, device="cuda", dtype=_TYPES[case["dtype"]]) for _ in range(2)]


def _table(used, ids, width):
    """Pages of every sequence, in a shuffled order; -1 behind its last one."""
    table = np.full((len(used), width), -1, np.int32)
    at = 0
    for s, u in enumerate(used):
        table[s, :u] = ids[at:at + u]
        at += u
    return table


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))
    st = {"case": case}
    op, seqs, heads, g, dim = case["op"], case["seqs"], case.get("q_heads", 0), case["kv_heads"], case["dim"]
    ctx = _spread(case, "ctx", seqs)
    nodes = _lengths(case)[1] if op != "evict" else np.zeros(seqs, np.int64)
    used = _pages_of(case, ctx + nodes)
    prefix_len = _spread(case, "prefix", case["prefixes"]) if op == "prefix" else np.zeros(0, np.int64)
    prefix_used = _pages_of(case, prefix_len)
    n_pages = int(used.sum() + prefix_used.sum()) + 3
    ids = rs.permutation(n_pages)
    st["k_pages"], st["v_pages"] = _cache(case, n_pages, gen)
    st["table"] = _gpu(_table(used, ids, int(used.max()) + 1))
    st["ctx_len"] = _gpu(ctx.astype(np.int32))
    if op == "evict":
        return _prepare_evict(case, st, gen, rs, ctx)
    row_begin = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    st["row_begin"] = _gpu(row_begin)
    st["live"], st["n_max"] = int(row_begin[-1]), int(nodes.max())
    n = st["n_tok"] = st["live"] + case.get("pad", 0)
    seq = np.minimum(np.searchsorted(row_begin[1:], np.arange(n), side="right"), seqs - 1)
    local = np.arange(n) - row_begin[seq]
    dt = _TYPES[case["dtype"]]
    if op == "norm":
        scale = torch.rand((n, heads + 2 * g, 1), generator=gen, device="cuda").mul_(4).exp_()      # heads of very different size
        st["qkv"] = torch.randn((n, heads + 2 * g, dim), generator=gen, device="cuda").mul_(scale).to(_TYPES[case["src"]])
        for name, h in (("q_gain", heads), ("k_gain", g)):
            st[name] = torch.randn((h, dim) if case["head_gain"] else (dim,), generator=gen, device="cuda").mul_(0.2).add_(1.0)
        st["q_out"] = torch.zeros((n, heads, dim), dtype=dt, device="cuda")
        axis, rank, axes = _axes(case["axes"], dim)
        # text counts on all axes; every other stretch of about 300 tokens is an image, whose rows and columns count from its start
        slot = ctx[seq] + local
        image = (slot // 300) % 2 == 1
        start, within = slot // 300 * 300, slot % 300
        pos = np.stack([np.where(image, start if a == 0 else start + (within // 20 if a == 1 else within % 20), slot) for a in range(3)])
        st["positions"] = _gpu(pos[3 - axes:].astype(np.int32))
        st["axis"], st["rank"] = torch.from_numpy(axis).cuda(), torch.from_numpy(rank).cuda()
    else:
        st["q"] = torch.randn((n, heads, dim), generator=gen, device="cuda").mul_(1.5).to(dt)
    if op == "prefix":
        st["prefix_table"] = _gpu(_table(prefix_used, ids[int(used.sum()):], int(prefix_used.max()) + 1))
        st["prefix_len"], st["seq_begin"] = _gpu(prefix_len.astype(np.int32)), _gpu(_groups(case))
        st["out"] = torch.zeros((n, heads, dim), dtype=dt, device="cuda")
        st["lse"] = torch.zeros((n, heads), dtype=torch.float32, device="cuda")
    if op == "weights":
        slots = int((ctx + nodes).max()) + 5
        x = _own_scores(st)[0]
        st["lse"] = torch.logsumexp(x, -1).permute(0, 3, 1, 2).reshape(seqs, -1, heads)[_gpu(seq), _gpu(local)].contiguous()      # as the attention left it
        del x
        # what the positions had received so far: a few much, most of them little
        st["weight"] = torch.randn((seqs, g, slots), generator=gen, device="cuda").mul_(2).exp_()
        st["weight_out"] = torch.zeros((seqs, g, slots), device="cuda")
        st["born"] = torch.arange(slots, dtype=torch.int32, device="cuda").repeat(seqs, g, 1)
        st["pos"] = _gpu((ctx[seq] + local + 1000).astype(np.int32))      # 1000 positions of the sequence have been dropped before
    if own:
        from paper_2504_08791_b200 import binding
        pool = st["pool"] = binding.PagedCache(st["k_pages"], st["v_pages"], rope_theta=_THETA, rope_mode=case.get("mode", 0))
        batch = st["batch"] = binding.PagedBatch(st["table"], st["row_begin"], st["ctx_len"], n, pos=st.get("pos"))
        if op == "norm":
            st["axes"] = binding.RopeAxes(axis.tolist(), rank.tolist())
        if op == "prefix":
            st["prefix"] = binding.PrefixBatch(st["prefix_table"], st["prefix_len"], st["seq_begin"])
            st["workspace"] = pool.prefix_attention_workspace(batch, st["prefix"], heads)
    return st


def _prepare_evict(case, st, gen, rs, ctx):
    seqs, g, layers = case["seqs"], case["kv_heads"], case["layers"]
    slots = int(ctx.max()) + 1
    shape = (layers, seqs, g, slots)
    st["weight"] = torch.randn(shape, generator=gen, device="cuda").mul_(2).exp_()
    # entries of an evicted and refilled cache: every slot holds some position, in no order
    st["born"] = torch.rand(shape, generator=gen, device="cuda").argsort(-1).int()
    st["weight_out"] = torch.zeros(shape, device="cuda")
    st["born_out"] = torch.zeros(shape, dtype=torch.int32, device="cuda")
    st["keep"] = _gpu(_spread(case, "keep", seqs)[::-1].astype(np.int32))
    st["recent_from"] = _gpu((slots - np.full(seqs, case["recent"])).astype(np.int32))
    st["length_out"] = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    if own:
        from paper_2504_08791_b200 import binding
        pool = st["pool"] = binding.PagedCache(st["k_pages"], st["v_pages"], rope_theta=_THETA)
        st["workspace"] = pool.evict_workspace(seqs, slots)
    return st


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _norm_own, "prefix": _prefix_own, "weights": _weights_own, "evict": _evict_own}[op](state)
    return {"norm": _norm_plain, "prefix": _prefix_plain, "weights": _weights_plain, "evict": _evict_plain}[op](state)


# ---- the package's entry points ---------------------------------------------------------------------
def _norm_own(s):
    h, g = s["case"]["q_heads"], s["case"]["kv_heads"]
    x = s["qkv"]
    s["pool"].append_norm(0, s["batch"], x[:, :h], x[:, h:h + g], x[:, h + g:], s["q_out"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=_EPS,
                          positions=s["positions"], axes=s["axes"])
    return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}


def _prefix_own(s):
    s["pool"].prefix_attention(0, s["batch"], s["prefix"], s["q"], s["out"], lse=s["lse"], workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _weights_own(s):
    case = s["case"]
    s["pool"].attention_weights(0, s["batch"], s["q"], s["lse"], s["weight_out"], weight_in=None if case["first_time"] else s["weight"],
                                decay=case["decay"], born=s["born"])
    return {"weight": s["weight_out"], "born": s["born"]}


def _evict_own(s):
    s["pool"].evict(s["table"], s["ctx_len"], s["weight"], s["born"], s["keep"], s["length_out"], weight_out=s["weight_out"], born_out=s["born_out"],
                    first=s["case"]["first"], recent_from=s["recent_from"], workspace=s["workspace"])
    return {"k": s["k_pages"], "v": s["v_pages"], "weight": s["weight_out"], "born": s["born_out"], "length": s["length_out"]}


# ---- plain forms ------------------------------------------------------------------------------------
def _seq_of(s, n):
    """Sequence and index within it of every row."""
    t = torch.arange(n, device="cuda")
    rb = s["row_begin"].long()
    seq = torch.searchsorted(rb[1:].contiguous(), t, right=True).clamp(max=rb.numel() - 2)
    return seq, t - rb[seq]


def _norm_plain(s):
    case = s["case"]
    h, g, dim, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    x = s["qkv"].float()

    def normed(y, gain):
        return y * torch.rsqrt((y * y).mean(-1, keepdim=True) + _EPS) * gain

    # angles in 64 bits: at far positions 32 would lose the fraction of a turn
    freq = torch.pow(_THETA, -2.0 * s["rank"].double() / dim)
    angle = s["positions"].double()[s["axis"].clamp(min=0)].T * freq * (s["axis"] >= 0)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(y):
        a, b = (y[..., :dim // 2], y[..., dim // 2:]) if case["mode"] == 0 else (y[..., 0::2], y[..., 1::2])
        u, v = a * cos - b * sin, a * sin + b * cos
        return torch.cat([u, v], -1) if case["mode"] == 0 else torch.stack([u, v], -1).flatten(-2)

    q, k = turned(normed(x[:, :h], s["q_gain"])), turned(normed(x[:, h:h + g], s["k_gain"]))
    m = s["live"]      # the rows of the sequences come first
    seq, local = _seq_of(s, m)
    slot = s["ctx_len"].long()[seq] + local
    at = s["table"].long()[seq, slot // page], slice(None), slot % page
    s["k_pages"][0][at] = k[:m].to(s["k_pages"].dtype)
    s["v_pages"][0][at] = x[:m, h + g:].to(s["v_pages"].dtype)
    s["q_out"][:m] = q[:m].to(s["q_out"].dtype)
    return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}


def _entries(s, table, which):
    """[sequences][KV heads][slots][head size] in 32 bits"""
    c = s[which][0][table.long().clamp(min=0)].float().permute(0, 2, 1, 3, 4)
    return c.reshape(c.shape[0], c.shape[1], -1, c.shape[-1])


def _padded_queries(s):
    """[sequences][KV heads][query heads of one][rows][head size]"""
    case = s["case"]
    rb = s["row_begin"].long()
    rows = (rb[:-1, None] + torch.arange(s["n_max"], device="cuda")).clamp(max=s["n_tok"] - 1)
    return s["q"].float()[rows].reshape(case["seqs"], s["n_max"], case["kv_heads"], -1, case["dim"]).permute(0, 2, 3, 1, 4)


def _own_scores(s):
    """[sequences][KV heads][query heads of one][rows][slots]: a row sees the positions in front of the step and the rows up to itself."""
    case = s["case"]
    k = _entries(s, s["table"], "k_pages")
    q = _padded_queries(s)
    x = torch.matmul(q.reshape(case["seqs"], case["kv_heads"], -1, case["dim"]), k.transpose(-1, -2)).reshape(*q.shape[:4], -1)
    rb, ctx = s["row_begin"].long(), s["ctx_len"].long()
    i, j = torch.arange(s["n_max"], device="cuda"), torch.arange(x.shape[-1], device="cuda")
    hidden = (j[None, None] > ctx[:, None, None] + i[None, :, None]) | (i[None] >= (rb[1:] - rb[:-1])[:, None])[..., None]
    return x.mul_(1 / math.sqrt(case["dim"])).masked_fill_(hidden[:, None, None], -math.inf), k


def _prefix_plain(s):
    case = s["case"]
    h, g, dim, m = case["q_heads"], case["kv_heads"], case["dim"], s["live"]
    seq, local = _seq_of(s, m)
    x, _ = _own_scores(s)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), _entries(s, s["table"], "v_pages")).reshape(*p.shape[:4], dim)

    def rows_of(y):
        return y.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, local]

    top, total, o = rows_of(top), rows_of(total), rows_of(o)                            # [rows][query heads][...]
    out, lse = s["out"].clone(), s["lse"].clone()
    group = torch.searchsorted(s["seq_begin"][1:].contiguous(), seq.int(), right=True)
    for i in range(case["prefixes"]):
        of = (group == i) & (seq >= s["seq_begin"][0])
        at = of.nonzero().flatten()
        j = torch.arange(s["prefix_table"].shape[1] * case["page"], device="cuda")
        q = s["q"].float()[at].reshape(-1, g, h // g, dim).transpose(0, 1)                    # [KV heads][rows][query heads of one][head size]
        y = torch.matmul(q.flatten(1, 2), _entries(s, s["prefix_table"][i:i + 1], "k_pages")[0].transpose(-1, -2)).mul_(1 / math.sqrt(dim))
        y.masked_fill_(j >= s["prefix_len"][i], -math.inf)

        def heads_of(z):
            return z.reshape(g, at.numel(), h // g, -1).transpose(0, 1).flatten(1, 2)

        t = y.amax(-1, keepdim=True)
        e = y.sub_(t).exp_()
        t, n, w = heads_of(t), heads_of(e.sum(-1, keepdim=True)), heads_of(torch.matmul(e, _entries(s, s["prefix_table"][i:i + 1], "v_pages")[0]))
        both = torch.maximum(t, top[at])
        a, b = (t - both).exp(), (top[at] - both).exp()
        n = n * a + total[at] * b
        out[at] = ((w * a + o[at] * b) / n).to(out.dtype)
        lse[at] = (both + n.log())[..., 0]
    return {"out": out, "lse": lse}


def _weights_plain(s):
    case = s["case"]
    ctx, rb = s["ctx_len"].long(), s["row_begin"].long()
    x, _ = _own_scores(s)
    rows = (rb[:-1, None] + torch.arange(s["n_max"], device="cuda")).clamp(max=s["n_tok"] - 1)
    lse = s["lse"][rows].reshape(case["seqs"], s["n_max"], case["kv_heads"], -1).permute(0, 2, 3, 1)
    p = x.sub_(lse[..., None]).exp_().flatten(2, 3).sum(2)                                       # [sequences][KV heads][slots]
    n = s["weight"].shape[-1]
    p = torch.nn.functional.pad(p, (0, max(0, n - p.shape[-1])))[..., :n]
    j = torch.arange(n, device="cuda")
    old = (j < ctx[:, None])[:, None]
    new = ((j >= ctx[:, None]) & (j < (ctx + rb[1:] - rb[:-1])[:, None]))[:, None]
    had = torch.zeros_like(p) if case["first_time"] else s["weight"] * case["decay"]
    weight = torch.where(old, had + p, torch.where(new, p, s["weight_out"]))
    came = s["pos"][(rb[:-1, None] + j - ctx[:, None]).clamp(0, s["n_tok"] - 1)][:, None]
    return {"weight": weight, "born": torch.where(new, came, s["born"])}


def _evict_plain(s):
    case = s["case"]
    layers, seqs, g, page = case["layers"], case["seqs"], case["kv_heads"], case["page"]
    n = s["weight"].shape[-1]
    j = torch.arange(n, device="cuda")
    there = (j < s["ctx_len"][:, None])[:, None]
    stays = (s["born"] < case["first"]) | (s["born"] >= s["recent_from"][:, None, None])
    key = torch.where(there, torch.where(stays, math.inf, s["weight"]), -math.inf)
    kept_n = torch.minimum(s["keep"], s["ctx_len"]).long()[:, None, None]
    order = key.sort(dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(key, dtype=torch.bool).scatter_(-1, order, (j < kept_n).expand_as(key))
    # the empty slots in front take the kept entries behind, each in ascending order
    hole, mover = ~kept & (j < kept_n), kept & (j >= kept_n)
    movers = torch.where(mover, j, n).sort(dim=-1).values
    source = torch.where(hole, movers.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0)), j)
    front = (j < kept_n).expand_as(key)
    weight = torch.where(front, s["weight"].gather(-1, source), s["weight_out"])
    born = torch.where(front, s["born"].gather(-1, source), s["born_out"])
    layer, q, head, to = hole.nonzero(as_tuple=True)
    come = source[layer, q, head, to]
    table = s["table"].long()
    for c in (s["k_pages"], s["v_pages"]):
        c[layer, table[q, to // page], head, to % page] = c[layer, table[q, come // page], head, come % page]
    return {"k": s["k_pages"], "v": s["v_pages"], "weight": weight, "born": born, "length": torch.minimum(s["keep"], s["ctx_len"])}


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    two = 2
    g, dim = case["kv_heads"], case["dim"]
    entry = 2 * g * dim * two          # key and value of one position
    if case["op"] == "evict":
        ctx = _spread(case, "ctx", case["seqs"])
        keep = np.minimum(_spread(case, "keep", case["seqs"])[::-1], ctx)
        # entries are chosen without regard to their slot: the part of the kept ones that lies behind the first `keep` moves
        moved = float((keep * (ctx - keep) / ctx).sum())
        per_layer = 2 * moved * entry + float((ctx * 8 + keep * 8).sum()) * g
        return {"bytes": int(case["layers"] * per_layer), "flops": 0}
    ctx, nodes = _lengths(case)
    n, heads = int(nodes.sum()), case["q_heads"]
    if case["op"] == "norm":
        src = torch.finfo(_TYPES[case["src"]]).bits // 8
        return {"bytes": n * ((heads + 2 * g) * dim * src + heads * dim * two + entry + 12), "flops": n * 7 * (heads + g) * dim}
    if case["op"] == "weights":
        total = int((ctx + nodes).sum())
        return {"bytes": total * (entry // 2 + g * (4 if case["first_time"] else 8)) + n * heads * (dim * two + 4),
                "flops": int((2 * heads * dim * nodes * (ctx + nodes)).sum())}
    prefix, begin = _spread(case, "prefix", case["prefixes"]), _groups(case)
    rows = np.array([nodes[begin[i]:begin[i + 1]].sum() for i in range(case["prefixes"])])
    return {"bytes": int(prefix.sum() + (ctx + nodes).sum()) * entry + n * heads * (2 * dim * two + 4),
            "flops": int(4 * heads * dim * ((nodes * (ctx + nodes)).sum() + (rows * prefix).sum()))}


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm_exact, "prefix": _prefix_exact, "weights": _weights_exact, "evict": _evict_exact}[case["op"]](case, s)


def _slots(case, table_row, first, count):
    """Page and row of the slots first .. first + count - 1 of one sequence."""
    j = np.arange(first, first + count)
    return torch.from_numpy(table_row[j // case["page"]].astype(np.int64)).cuda(), torch.from_numpy(j % case["page"]).cuda()


def _norm_exact(case, s):
    h, g, dim = case["q_heads"], case["kv_heads"], case["dim"]
    x = s["qkv"].double()
    gain = torch.cat([s["q_gain"].expand(h, dim), s["k_gain"].expand(g, dim)]).double()
    y = x[:, :h + g]
    y = gain * y / torch.sqrt(torch.linalg.vector_norm(y, dim=-1, keepdim=True) ** 2 / dim + _EPS)
    axis, rank, _ = _axes(case["axes"], dim)
    positions = s["positions"].double()
    angle = torch.stack([positions[a] * math.exp(-2 * math.log(_THETA) * r / dim) if a >= 0 else torch.zeros_like(positions[0]) for a, r in zip(axis, rank)], -1)
    z = torch.polar(torch.ones_like(angle), angle)
    pair = y.unflatten(-1, (2, dim // 2)).transpose(-1, -2) if case["mode"] == 0 else y.unflatten(-1, (dim // 2, 2))
    turned = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z[:, None])
    turned = (turned.transpose(-1, -2) if case["mode"] == 0 else turned).reshape(x.shape[0], h + g, dim)
    q, k, v = s["q_out"].double(), s["k_pages"].double(), s["v_pages"].double()
    table, rb, ctx = s["table"].cpu().numpy(), s["row_begin"].tolist(), s["ctx_len"].tolist()
    for i in range(case["seqs"]):
        page, row = _slots(case, table[i], ctx[i], rb[i + 1] - rb[i])
        k[0, page, :, row] = turned[rb[i]:rb[i + 1], h:]
        v[0, page, :, row] = x[rb[i]:rb[i + 1], h + g:]
    q[:rb[-1]] = turned[:rb[-1], :h]
    return {"q": q, "k": k, "v": v}


def _prefix_exact(case, s):
    h, g, dim = case["q_heads"], case["kv_heads"], case["dim"]
    out, lse = s["out"].double(), s["lse"].double()
    table, rb, ctx = s["table"].cpu().numpy(), s["row_begin"].tolist(), s["ctx_len"].tolist()
    of_prefix, begin, length = s["prefix_table"].cpu().numpy(), s["seq_begin"].tolist(), s["prefix_len"].tolist()
    for p in range(case["prefixes"]):
        page, row = _slots(case, of_prefix[p], 0, length[p])
        for kv in range(g):
            at = slice(kv * (h // g), (kv + 1) * (h // g))
            pk, pv = (c[0, page, kv, row].double() for c in (s["k_pages"], s["v_pages"]))
            for first in range(begin[p], begin[p + 1], 16):      # sixteen sequences at a time share the product with the prefix
                last = min(first + 16, begin[p + 1])
                q = s["q"][rb[first]:rb[last], at].double()
                far = torch.einsum("nhd,ld->nhl", q, pk) / dim ** 0.5
                for i in range(first, last):
                    mine = slice(rb[i] - rb[first], rb[i + 1] - rb[first])
                    n = rb[i + 1] - rb[i]
                    own_page, own_row = _slots(case, table[i], 0, ctx[i] + n)
                    k, v = (c[0, own_page, kv, own_row].double() for c in (s["k_pages"], s["v_pages"]))
                    near = torch.einsum("nhd,ld->nhl", q[mine], k) / dim ** 0.5
                    behind = torch.arange(ctx[i] + n, device="cuda")[None] - ctx[i] > torch.arange(n, device="cuda")[:, None]
                    near = near.masked_fill(behind[:, None], -math.inf)
                    x = torch.cat([far[mine], near], -1)
                    z = torch.logsumexp(x, -1)
                    out[rb[i]:rb[i + 1], at] = torch.einsum("nhl,ld->nhd", torch.exp(x - z[..., None]), torch.cat([pv, v]))
                    lse[rb[i]:rb[i + 1], at] = z
    return {"out": out, "lse": lse}


def _weights_exact(case, s):
    h, g, dim = case["q_heads"], case["kv_heads"], case["dim"]
    weight = s["weight_out"].double()
    table, rb, ctx = s["table"].cpu().numpy(), s["row_begin"].tolist(), s["ctx_len"].tolist()
    for i in range(case["seqs"]):
        n = rb[i + 1] - rb[i]
        page, row = _slots(case, table[i], 0, ctx[i] + n)
        behind = torch.arange(ctx[i] + n, device="cuda")[None] - ctx[i] > torch.arange(n, device="cuda")[:, None]
        for kv in range(g):
            at = slice(kv * (h // g), (kv + 1) * (h // g))
            x = torch.einsum("nhd,ld->nhl", s["q"][rb[i]:rb[i + 1], at].double(), s["k_pages"][0, page, kv, row].double()) / dim ** 0.5
            x = x.masked_fill(behind[:, None], -math.inf) - s["lse"][rb[i]:rb[i + 1], at, None].double()
            sums = torch.exp(x).sum((0, 1))
            if not case["first_time"]:
                sums[:ctx[i]] += case["decay"] * s["weight"][i, kv, :ctx[i]].double()
            weight[i, kv, :ctx[i] + n] = sums
    return {"weight": weight, "born": None}


def _evict_exact(case, s):
    page = case["page"]
    table, ctx, keep, recent = (s[x].cpu().numpy() for x in ("table", "ctx_len", "keep", "recent_from"))
    weight, born = s["weight"].cpu().numpy(), s["born"].cpu().numpy()
    weight_out, born_out = s["weight_out"].cpu().numpy().astype(np.float64), s["born_out"].cpu().numpy()
    to, come = [], []
    for index in np.ndindex(case["layers"], case["seqs"], case["kv_heads"]):
        layer, i, head = index
        n = int(ctx[i])
        m = min(n, int(keep[i]))
        w, b = weight[index][:n].astype(np.float64), born[index][:n]
        w = np.where((b < case["first"]) | (b >= recent[i]), np.inf, w)
        kept = np.sort(np.lexsort((np.arange(n), -w))[:m])
        source = np.arange(m)
        holes = np.setdiff1d(source, kept)
        source[holes] = kept[kept >= m]
        weight_out[index][:m], born_out[index][:m] = weight[index][source], born[index][source]
        for where, slot in ((to, holes), (come, source[holes])):
            where.append(np.stack([np.full(slot.size, layer), table[i, slot // page], np.full(slot.size, head), slot % page]))
    to, come = (torch.from_numpy(np.concatenate(x, 1)).long().cuda() for x in (to, come))
    k, v = s["k_pages"].clone(), s["v_pages"].clone()
    for c in (k, v):
        c[tuple(to)] = c[tuple(come)]
    return {"k": k, "v": v, "weight": torch.from_numpy(weight_out).cuda(), "born": None, "length": None}
