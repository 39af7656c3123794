"""The operators for several candidate continuations of a sequence over one paged cache, as cases to be measured.

  append   rotary position encoding of queries and keys, keys and values appended to a paged cache
  tree     attention of drafted token trees (or chains, or single tokens) over the paged cache
  accept   the entries of an accepted path of the tree moved to the positions that follow the context
  beam     the best continuations of beams over the vocabulary, and the reordering of their caches' page tables

``run`` computes each in plain torch operations, or, where ``own`` is true, by the package's entry points.
Cache layout: [layers][pages][KV heads][page size][head size]; sequence s holds position j in page
table[s][j // page size] at row j % page size.  Lengths follow from the case alone, values from the seed.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _cases():
    return [
        # one token of one request enters the cache, 8B-shaped heads: what a decoding step pays per layer
        {"name": "append_one", "op": "append", "dtype": "f16", "src": "f32", "seqs": 1, "nodes": [1, 1], "ctx": [1024, 1024],
         "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "mode": 0, "layers": 1, "pad": 0},
        # drafted trees of a batch of requests, 70B-shaped heads, ragged, rotation of neighbouring pairs, two padded rows
        {"name": "append_trees", "op": "append", "dtype": "f16", "src": "f16", "seqs": 32, "nodes": [1, 25], "ctx": [17, 4000],
         "q_heads": 64, "kv_heads": 8, "dim": 128, "page": 32, "mode": 1, "layers": 1, "pad": 2},
        # prompts of four requests enter the cache at once, 32B-shaped heads
        {"name": "append_prompts", "op": "append", "dtype": "bf16", "src": "bf16", "seqs": 4, "nodes": [1500, 4096], "ctx": [0, 0],
         "q_heads": 40, "kv_heads": 8, "dim": 128, "page": 64, "mode": 0, "layers": 1, "pad": 0},
        # the smallest verification: four drafted tokens and the newest one over a short context, 8B-shaped heads
        {"name": "tree_small", "op": "tree", "dtype": "f16", "seqs": 1, "nodes": [5, 5], "ctx": [1000, 1000],
         "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "mask": True, "layers": 1, "pad": 0},
        # single tokens of a batch of requests (no tree): the serving step, heads of 64
        {"name": "tree_decode", "op": "tree", "dtype": "bf16", "seqs": 64, "nodes": [1, 1], "ctx": [1, 4096],
         "q_heads": 32, "kv_heads": 8, "dim": 64, "page": 16, "mask": False, "layers": 1, "pad": 0},
        # ragged trees of a batch of requests, 32B-shaped heads (five query heads share a KV head), padded rows behind them
        {"name": "tree_batch", "op": "tree", "dtype": "bf16", "seqs": 16, "nodes": [1, 26], "ctx": [100, 8192],
         "q_heads": 40, "kv_heads": 8, "dim": 128, "page": 32, "mask": True, "layers": 1, "pad": 3},
        # a tree of 64 nodes over a long context, 70B-shaped heads
        {"name": "tree_long", "op": "tree", "dtype": "f16", "seqs": 1, "nodes": [64, 64], "ctx": [65531, 65531],
         "q_heads": 64, "kv_heads": 8, "dim": 128, "page": 64, "mask": True, "layers": 1, "pad": 0},
        # one request's accepted path (up to five tokens), all 32 layers of an 8B-shaped model
        {"name": "accept_one", "op": "accept", "dtype": "f16", "seqs": 1, "nodes": [16, 16], "path": [4, 4], "ctx": [1021, 1021],
         "kv_heads": 8, "dim": 128, "page": 16, "layers": 32},
        # accepted paths of a batch of requests, all 80 layers of a 70B-shaped model
        {"name": "accept_batch", "op": "accept", "dtype": "bf16", "seqs": 32, "nodes": [1, 64], "path": [1, 12], "ctx": [3, 700],
         "kv_heads": 8, "dim": 128, "page": 32, "layers": 80},
        # four beams of one request, small vocabulary, shallow model
        {"name": "beam_small", "op": "beam", "dtype": "f16", "logits": "f32", "reqs": 1, "beams": 4, "keep": 4, "vocab": 32000,
         "finished": False, "ctx": [37, 37], "kv_heads": 8, "dim": 128, "page": 16, "layers": 32},
        # three requests of eight beams, 32B-shaped: some have ended, an odd vocabulary in 16 bits
        {"name": "beam_half", "op": "beam", "dtype": "bf16", "logits": "bf16", "reqs": 3, "beams": 8, "keep": 8, "vocab": 128259,
         "finished": True, "ctx": [5, 200], "kv_heads": 8, "dim": 128, "page": 16, "layers": 64},
        # sixteen requests of eight beams, the 32B shape's vocabulary
        {"name": "beam_large", "op": "beam", "dtype": "f16", "logits": "f32", "reqs": 16, "beams": 8, "keep": 8, "vocab": 152064,
         "finished": True, "ctx": [16, 300], "kv_heads": 8, "dim": 128, "page": 16, "layers": 16},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    def span(lo, hi):
        a, b = log(lo, hi), log(lo, hi)
        return [min(a, b), max(a, b)]

    op = rng.choice(["append", "tree", "tree", "accept", "beam"])
    case = {"op": op, "dtype": rng.choice(["f16", "bf16"]), "dim": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128]),
            "kv_heads": rng.choice([1, 2, 4, 8])}
    group = rng.choice([1, 2, 3, 4, 5, 7, 8])
    if op == "append":
        seqs = log(1, 64)
        case |= {"src": rng.choice(["f32", case["dtype"]]), "seqs": seqs, "nodes": span(1, max(1, 6000 // seqs)), "ctx": span(1, 4096),
                 "mode": rng.choice([0, 1]), "layers": 1, "pad": rng.choice([0, 0, 5])}
    elif op == "tree":
        seqs = log(1, 64)
        top = max(16, 65536 // seqs)
        case |= {"seqs": seqs, "nodes": span(1, max(1, min(64, 400 // seqs))), "ctx": span(1, top), "mask": rng.random() < 0.75,
                 "layers": rng.choice([1, 2]), "pad": rng.choice([0, 0, 3])}
    elif op == "accept":
        case |= {"seqs": log(1, 24), "nodes": span(1, 64), "path": span(1, 12), "ctx": span(1, 700), "layers": log(1, 80)}
    else:
        beams = rng.randint(1, 16)
        case |= {"logits": rng.choice(["f32", "f32", "f16", "bf16"]), "reqs": log(1, 16), "beams": beams, "keep": rng.randint(1, beams),
                 "vocab": log(200, 152064), "finished": rng.random() < 0.5, "ctx": span(1, 300), "layers": log(1, 16)}
        while case["reqs"] * beams * case["vocab"] > 16 * 8 * 152064:
            case["reqs"] //= 2
    if op in ("append", "tree"):
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


def _pages_of(case, lengths):
    return -(-lengths // case["page"])


def _lengths(case):
    """(tokens of the context, tokens of the step) of every sequence."""
    return _spread(case, "ctx", case["seqs"]), _spread(case, "nodes", case["seqs"])[::-1].copy()


def _cache(case, n_pages, gen):
    shape = (case["layers"], n_pages, case["kv_heads"], case["page"], case["dim"])
    dt = _TYPES[case["dtype"]]
    return [torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dt) if math.prod(shape) < 1 << 28
            else torch.randn(shape, generator=gen, device="cuda", dtype=dt) for _ in range(2)]


def _table(case, used, n_pages, rs, width):
    """Pages of every sequence, in a shuffled order; -1 behind its last one."""
    ids = rs.permutation(n_pages)[: int(used.sum())]
    table = np.full((len(used), width), -1, np.int32)
    at = 0
    for s, u in enumerate(used):
        table[s, :u] = ids[at:at + u]
        at += u
    return table


def _trees(case, nodes, rs):
    """Random trees: every node's ancestors and itself as bits of a 64-bit word, and its depth."""
    bits, depth = [], []
    for n in nodes:
        b, d = [], []
        for i in range(n):
            p = int(rs.randint(max(0, i - 6), i)) if i else -1
            b.append((b[p] if i else 0) | 1 << i)
            d.append(d[p] + 1 if i else 0)
        bits += b
        depth += d
    return np.array(bits, np.uint64).view(np.int64), np.array(depth, np.int32)


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 32))
    st = {"case": case}
    if case["op"] == "beam":
        return _prepare_beam(case, st, gen, rs)
    ctx, nodes = _lengths(case)
    used = _pages_of(case, ctx + nodes)
    n_pages = int(used.sum()) + 3
    st["k_pages"], st["v_pages"] = _cache(case, n_pages, gen)
    st["table"] = _gpu(_table(case, used, n_pages, rs, int(used.max()) + 1))
    st["ctx_len"] = _gpu(ctx.astype(np.int32))
    row_begin = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    st["row_begin"] = _gpu(row_begin)
    st["layer"] = case["layers"] - 1
    n = int(row_begin[-1])
    if case["op"] == "accept":
        path_len = np.minimum(_spread(case, "path", case["seqs"]), nodes)
        path = np.zeros((case["seqs"], int(path_len.max())), np.int32)
        for s in range(case["seqs"]):
            path[s, :path_len[s]] = np.sort(rs.permutation(nodes[s])[:path_len[s]])
        st["path"], st["path_len"] = _gpu(path), _gpu(path_len.astype(np.int32))
    else:
        n += case["pad"]
        st["n_tok"], st["n_max"] = n, int(nodes.max())
        dt, dim, heads = _TYPES[case["dtype"]], case["dim"], case["q_heads"]
        seq = np.minimum(np.searchsorted(row_begin[1:], np.arange(n), side="right"), case["seqs"] - 1)
        local = np.arange(n) - row_begin[seq]
        if case["op"] == "append":
            src = _TYPES[case["src"]]
            st["qkv"] = torch.randn((n, heads + 2 * case["kv_heads"], dim), generator=gen, device="cuda").to(src)
            st["q_out"] = torch.zeros((n, heads, dim), dtype=dt, device="cuda")
            # within a tree several tokens share a position: a token sits at most at its index behind the context
            st["pos"] = _gpu((ctx[seq] + np.maximum(0, local - rs.randint(0, 3, n) * (case["nodes_max"] <= 64))).astype(np.int32))
        else:
            st["q"] = torch.randn((n, heads, dim), generator=gen, device="cuda").mul_(1.5).to(dt)
            st["out"] = torch.zeros((n, heads, dim), dtype=dt, device="cuda")
            st["lse"] = torch.zeros((n, heads), dtype=torch.float32, device="cuda")
            if case["mask"]:
                mask = np.zeros(n, np.int64)
                mask[: int(row_begin[-1])] = _trees(case, nodes, rs)[0]
                st["mask"] = _gpu(mask.reshape(n, 1))
    if own:
        from paper_2504_08791_b200 import binding
        st["pool"] = binding.PagedCache(st["k_pages"], st["v_pages"], rope_theta=5e5, rope_mode=case.get("mode", 0))
        st["batch"] = binding.PagedBatch(st["table"], st["row_begin"], st["ctx_len"], st.get("n_tok", n), pos=st.get("pos"), mask=st.get("mask"))
        if case["op"] == "tree":
            st["workspace"] = st["pool"].tree_attention_workspace(st["batch"])
    return st


def _prepare_beam(case, st, gen, rs):
    reqs, beams, keep, page = case["reqs"], case["beams"], case["keep"], case["page"]
    length = np.repeat(_spread(case, "ctx", reqs), beams)
    used = _pages_of(case, length)
    n_pages = int(used.sum()) + reqs * keep + 3
    st["k_pages"], st["v_pages"] = _cache(case, n_pages, gen)
    table = _table(case, used, n_pages - reqs * keep, rs, int(used.max()) + 1)
    st["table"], st["length"] = _gpu(table), _gpu(length.astype(np.int32))
    st["fresh"] = _gpu((n_pages - reqs * keep + rs.permutation(reqs * keep)).astype(np.int32))
    st["table_out"] = torch.zeros((reqs * keep, table.shape[1]), dtype=torch.int32, device="cuda")
    st["length_out"] = torch.zeros(reqs * keep, dtype=torch.int32, device="cuda")
    logits = torch.randn((reqs, beams, case["vocab"]), generator=gen, device="cuda").mul_(2.5)
    # a sampler's filter has taken some words out
    logits.masked_fill_(torch.rand(case["vocab"], generator=gen, device="cuda") < 0.01, -math.inf)
    st["logits"] = logits.to(_TYPES[case["logits"]])
    st["cum"] = _gpu(-np.sort(rs.gamma(4.0, 1.0, (reqs, beams)), axis=1).astype(np.float32))
    st["finished"] = _gpu((rs.rand(reqs, beams) < 0.25).astype(np.uint8)) if case["finished"] else None
    st["end"] = 2
    for name, dt in (("score", torch.float32), ("parent", torch.int32), ("token", torch.int32)):
        st[name] = torch.zeros((reqs, keep), dtype=dt, device="cuda")
    if own:
        from paper_2504_08791_b200 import binding
        st["pool"] = binding.PagedCache(st["k_pages"], st["v_pages"], rope_theta=5e5)
        st["workspace"] = binding.prima_beam_select_workspace(reqs, beams, case["vocab"], keep)
    return st


def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _append_own, "tree": _tree_own, "accept": _accept_own, "beam": _beam_own}[op](state)
    return {"append": _append_plain, "tree": _tree_plain, "accept": _accept_plain, "beam": _beam_plain}[op](state)


# ---- the package's entry points ---------------------------------------------------------------------
def _append_own(s):
    h, g = s["case"]["q_heads"], s["case"]["kv_heads"]
    x = s["qkv"]
    s["pool"].append(s["layer"], s["batch"], x[:, :h], x[:, h:h + g], x[:, h + g:], s["q_out"])
    return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}


def _tree_own(s):
    s["pool"].tree_attention(s["layer"], s["batch"], s["q"], s["out"], lse=s["lse"], workspace=s["workspace"])
    return {"out": s["out"], "lse": s["lse"]}


def _accept_own(s):
    s["pool"].accept(s["batch"], s["path"], s["path_len"])
    return {"k": s["k_pages"], "v": s["v_pages"]}


def _beam_own(s):
    from paper_2504_08791_b200 import binding
    binding.prima_beam_select(s["logits"], s["cum"], s["score"], s["parent"], s["token"], finished=s["finished"], end_token=s["end"],
                        workspace=s["workspace"])
    s["pool"].reorder(s["table"], s["length"], s["parent"], s["fresh"], s["table_out"], s["length_out"])
    return {"score": s["score"], "parent": s["parent"], "token": s["token"], "table": s["table_out"], "length": s["length_out"],
            "k": s["k_pages"], "v": s["v_pages"]}


# ---- plain forms ------------------------------------------------------------------------------------
def _seq_of(s, n):
    """Sequence and index within it of every row, and whether the row belongs to a sequence at all."""
    t = torch.arange(n, device="cuda")
    rb = s["row_begin"].long()
    seq = torch.searchsorted(rb[1:].contiguous(), t, right=True).clamp(max=rb.numel() - 2)
    return seq, t - rb[seq], t < rb[-1]


def _rotate(x, cos, sin, mode):
    """Pairs (i, i + dim/2) in mode 0, (2i, 2i + 1) in mode 1, turned by the angle of each row."""
    half = x.shape[-1] // 2
    a, b = (x[..., :half], x[..., half:]) if mode == 0 else (x[..., 0::2], x[..., 1::2])
    cos, sin = cos[:, None], sin[:, None]
    u, v = a * cos - b * sin, a * sin + b * cos
    return torch.cat([u, v], -1) if mode == 0 else torch.stack([u, v], -1).flatten(-2)


def _append_plain(s):
    case = s["case"]
    h, g, dim, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    seq, local, live = _seq_of(s, s["n_tok"])
    slot = s["ctx_len"].long()[seq] + local
    # angles in 64 bits: at far positions 32 would lose the fraction of a turn
    freq = torch.pow(5e5, -2.0 * torch.arange(dim // 2, device="cuda", dtype=torch.float64) / dim)
    angle = s["pos"].double()[:, None] * freq
    cos, sin = angle.cos().float(), angle.sin().float()
    x = s["qkv"].float()
    q, k = _rotate(x[:, :h], cos, sin, case["mode"]), _rotate(x[:, h:h + g], cos, sin, case["mode"])
    n = int(case["pad"])
    m = s["n_tok"] - n      # the rows of the sequences come first
    at = s["table"].long()[seq, slot // page][:m], slice(None), (slot % page)[:m]
    s["k_pages"][s["layer"]][at] = k[:m].to(s["k_pages"].dtype)
    s["v_pages"][s["layer"]][at] = x[:m, h + g:].to(s["v_pages"].dtype)
    s["q_out"][:m] = q[:m].to(s["q_out"].dtype)
    return {"q": s["q_out"], "k": s["k_pages"], "v": s["v_pages"]}


def _visible(s, length):
    """[sequences][rows][slots]: whether a row sees a slot of its sequence."""
    rb, ctx = s["row_begin"].long(), s["ctx_len"].long()
    i = torch.arange(s["n_max"], device="cuda")
    j = torch.arange(length, device="cuda")
    behind = j[None] - ctx[:, None]                                   # index in the tree of every slot
    nodes = (rb[1:] - rb[:-1])[:, None]
    if "mask" in s:
        word = s["mask"][:, 0][(rb[:-1, None] + i).clamp(max=s["n_tok"] - 1)]
        bit = (word[:, :, None] >> behind.clamp(0, 63)[:, None]) & 1
        seen = (bit != 0) & ((behind >= 0) & (behind < nodes) & (behind < 64))[:, None]
    else:
        seen = (behind >= 0)[:, None] & (behind[:, None] <= i[None, :, None])
    return seen | (behind < 0)[:, None]


def _tree_plain(s):
    case = s["case"]
    h, g, dim = case["q_heads"], case["kv_heads"], case["dim"]
    n_seq = case["seqs"]
    seq, local, live = _seq_of(s, s["n_tok"])
    pages = s["table"].long().clamp(min=0)
    k, v = (c[s["layer"]][pages].float().permute(0, 2, 1, 3, 4).reshape(n_seq, g, -1, dim) for c in (s["k_pages"], s["v_pages"]))
    rb = s["row_begin"].long()
    rows = (rb[:-1, None] + torch.arange(s["n_max"], device="cuda")).clamp(max=s["n_tok"] - 1)
    q = s["q"].float()[rows].reshape(n_seq, s["n_max"], g, h // g, dim).permute(0, 2, 3, 1, 4)
    score = torch.matmul(q.reshape(n_seq, g, -1, dim), k.transpose(-1, -2)).reshape(n_seq, g, h // g, s["n_max"], -1)
    score = score.mul_(1 / math.sqrt(dim)).masked_fill_(~_visible(s, k.shape[2])[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.reshape(n_seq, g, -1, p.shape[-1]), v).reshape(n_seq, g, h // g, s["n_max"], dim)
    out = out / torch.where(total == 0, torch.ones_like(total), total)
    lse = (top + total.log()).squeeze(-1)
    out = out.permute(0, 3, 1, 2, 4).reshape(n_seq, -1, h, dim)[seq, local.clamp(max=s["n_max"] - 1)]
    lse = lse.permute(0, 3, 1, 2).reshape(n_seq, -1, h)[seq, local.clamp(max=s["n_max"] - 1)]
    return {"out": torch.where(live[:, None, None], out, s["out"].float()).to(s["out"].dtype), "lse": torch.where(live[:, None], lse, s["lse"])}


def _accept_plain(s):
    page = s["case"]["page"]
    j = torch.arange(s["path"].shape[1], device="cuda")[None]
    to = s["ctx_len"].long()[:, None] + j
    come = torch.where(j < s["path_len"].long()[:, None], s["ctx_len"].long()[:, None] + s["path"].long(), to)
    table = s["table"].long()
    last = table.shape[1] * page - 1
    to, come = to.clamp(max=last), come.clamp(max=last)
    # a place behind the path that has no page is nobody's: it is left out by copying page -1 (the last, unused one) onto itself
    at = [(table.gather(1, x // page), x % page) for x in (to, come)]
    for c in (s["k_pages"], s["v_pages"]):
        c[:, at[0][0], :, at[0][1]] = c[:, at[1][0], :, at[1][1]]
    return {"k": s["k_pages"], "v": s["v_pages"]}


def _beam_plain(s):
    case = s["case"]
    reqs, beams, keep, vocab, page = case["reqs"], case["beams"], case["keep"], case["vocab"], case["page"]
    # in 64 bits: which of two near candidates is ahead is decided by the last bits
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    x = x - top
    x = x - x.exp().sum(-1, keepdim=True).log()
    x = x + s["cum"].double()[..., None]
    if s["finished"] is not None:
        done = s["finished"].bool()[..., None]
        word = torch.arange(vocab, device="cuda") == s["end"]
        x = torch.where(done, torch.where(word, s["cum"].double()[..., None], -math.inf), x)
    score, at = x.reshape(reqs, -1).sort(dim=-1, descending=True, stable=True)
    score, at = score[:, :keep], at[:, :keep]
    none = score == -math.inf
    parent = torch.where(none, 0, at // vocab).int()
    token = torch.where(none, -1, at % vocab).int()
    row = (torch.arange(reqs, device="cuda")[:, None] * beams + parent).flatten()
    length = s["length"][row]
    # the first child of a beam goes on in its last page; every other one gets a copy of the entries in it
    older = (row[:, None] == row[None]) & (torch.arange(row.numel(), device="cuda")[:, None] > torch.arange(row.numel(), device="cuda")[None])
    copied = older.any(1) & (length % page != 0)
    col = torch.arange(s["table"].shape[1], device="cuda")[None]
    table = torch.where(col < -(-length // page)[:, None], s["table"][row], -1)
    last = (length // page).long()
    source = table.gather(1, last[:, None].clamp(max=table.shape[1] - 1))[:, 0].long().clamp(min=0)
    table = torch.where(copied[:, None] & (col == last[:, None]), s["fresh"][:, None], table)
    moved = (copied[:, None] & (torch.arange(page, device="cuda")[None] < (length % page)[:, None]))[None, :, None, :, None]
    for c in (s["k_pages"], s["v_pages"]):
        c[:, s["fresh"].long()] = torch.where(moved, c[:, source], c[:, s["fresh"].long()])
    return {"score": score.float(), "parent": parent, "token": token, "table": table.int(), "length": length, "k": s["k_pages"], "v": s["v_pages"]}


# ---- what a pass cannot do without ------------------------------------------------------------------
def work(case):
    two = 2
    if case["op"] == "beam":
        size = torch.finfo(_TYPES[case["logits"]]).bits // 8
        n = case["reqs"] * case["beams"] * case["vocab"]
        rows = case["reqs"] * case["keep"]
        # about a third of the kept beams share a parent: their last pages' entries are read and written
        tails = _spread(case, "ctx", case["reqs"]) % case["page"]
        copied = int(tails.sum()) * case["keep"] // 3
        entry = 2 * case["layers"] * case["kv_heads"] * case["dim"] * two
        return {"bytes": n * size + rows * 12 + 2 * copied * entry, "flops": 4 * n}
    ctx, nodes = _lengths(case)
    n = int(nodes.sum())
    entry = 2 * case["kv_heads"] * case["dim"] * two          # key and value of one position
    if case["op"] == "accept":
        moved = int(np.minimum(_spread(case, "path", case["seqs"]), nodes).sum())
        return {"bytes": 2 * moved * entry * case["layers"], "flops": 0}
    heads, dim = case["q_heads"], case["dim"]
    if case["op"] == "append":
        src = torch.finfo(_TYPES[case["src"]]).bits // 8
        return {"bytes": n * ((heads + 2 * case["kv_heads"]) * dim * src + heads * dim * two + entry + 4), "flops": n * 3 * (heads + case["kv_heads"]) * dim}
    return {"bytes": int((ctx + nodes).sum()) * entry + n * heads * (2 * dim * two + 4), "flops": int((4 * heads * dim * nodes * (ctx + nodes)).sum())}


# ---- the definitions in 64 bits ---------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _append_exact, "tree": _tree_exact, "accept": _accept_exact, "beam": _beam_exact}[case["op"]](case, s)


def _slots(case, table_row, first, count):
    """Page and row of the slots first .. first + count - 1 of one sequence."""
    j = np.arange(first, first + count)
    return torch.from_numpy(table_row[j // case["page"]].astype(np.int64)).cuda(), torch.from_numpy(j % case["page"]).cuda()


def _append_exact(case, s):
    h, g, dim = case["q_heads"], case["kv_heads"], case["dim"]
    x = s["qkv"].double()
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                    torch.outer(s["pos"].double(), torch.exp(-math.log(5e5) * torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)))
    pair = x[:, :h + g].unflatten(-1, (2, dim // 2)).transpose(-1, -2) if case["mode"] == 0 else x[:, :h + g].unflatten(-1, (dim // 2, 2))
    turned = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z[:, None])
    turned = (turned.transpose(-1, -2) if case["mode"] == 0 else turned).reshape(x.shape[0], h + g, dim)
    q, k, v = s["q_out"].double(), s["k_pages"].double(), s["v_pages"].double()
    table, rb, ctx = s["table"].cpu().numpy(), s["row_begin"].tolist(), s["ctx_len"].tolist()
    for i in range(case["seqs"]):
        page, row = _slots(case, table[i], ctx[i], rb[i + 1] - rb[i])
        k[s["layer"], page, :, row] = turned[rb[i]:rb[i + 1], h:]
        v[s["layer"], page, :, row] = x[rb[i]:rb[i + 1], h + g:]
    q[:rb[-1]] = turned[:rb[-1], :h]
    return {"q": q, "k": k, "v": v}


def _tree_exact(case, s):
    h, g, dim = case["q_heads"], case["kv_heads"], case["dim"]
    out, lse = s["out"].double(), s["lse"].double()
    table, rb, ctx = s["table"].cpu().numpy(), s["row_begin"].tolist(), s["ctx_len"].tolist()
    masks = s["mask"].cpu().numpy().view(np.uint64)[:, 0] if case["mask"] else None
    for i in range(case["seqs"]):
        n = rb[i + 1] - rb[i]
        page, row = _slots(case, table[i], 0, ctx[i] + n)
        see = np.ones((n, ctx[i] + n), bool)
        for a in range(n):
            see[a, ctx[i]:] = [(int(masks[rb[i] + a]) >> b) & 1 if masks is not None else b <= a for b in range(n)]
        see = torch.from_numpy(see).cuda()
        for kv in range(g):
            k, v = (c[s["layer"], page, kv, row].double() for c in (s["k_pages"], s["v_pages"]))
            q = s["q"][rb[i]:rb[i + 1], kv * (h // g):(kv + 1) * (h // g)].double()
            x = torch.einsum("nhd,ld->nhl", q, k) / dim ** 0.5
            x[~see[:, None].expand_as(x)] = -math.inf
            z = torch.logsumexp(x, -1)
            out[rb[i]:rb[i + 1], kv * (h // g):(kv + 1) * (h // g)] = torch.einsum("nhl,ld->nhd", torch.exp(x - z[..., None]), v)
            lse[rb[i]:rb[i + 1], kv * (h // g):(kv + 1) * (h // g)] = z
    return {"out": out, "lse": lse}


def _accept_exact(case, s):
    table, ctx, path, n = s["table"].cpu().numpy(), s["ctx_len"].tolist(), s["path"].cpu().numpy(), s["path_len"].tolist()
    got = {}
    for name in ("k_pages", "v_pages"):
        old = s[name]
        new = old.clone()
        for i in range(case["seqs"]):
            for j in range(n[i]):
                a, b = ctx[i] + int(path[i, j]), ctx[i] + j
                new[:, table[i, b // case["page"]], :, b % case["page"]] = old[:, table[i, a // case["page"]], :, a % case["page"]]
        got[name[0]] = new.double()
    return got


def _beam_exact(case, s):
    """Which candidates are chosen are whole numbers, compared as such: here are the scores of the best ones, in their order."""
    x = torch.log_softmax(s["logits"].double(), -1) + s["cum"].double()[..., None]
    if s["finished"] is not None:
        done = s["finished"].bool()
        x[done] = -math.inf
        x[..., s["end"]][done] = s["cum"].double()[done]
    score = x.flatten(1).topk(case["keep"], -1).values
    return {"score": score, "parent": None, "token": None, "table": None, "length": None, "k": None, "v": None}
