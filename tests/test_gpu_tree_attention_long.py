"""Tree attention where a CTA takes several consecutive units of a segment: references that move while the output is being
summed, in both kernels and for tiles of one and of two accumulators, against softmax in 64 bits."""
import numpy as np
import pytest

from tests import _paged
from tests._paged import Batch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

# nodes of a sequence (with 4 query heads per KV head) and positions: the streaming kernel; one accumulator; two; three
# tiles of 256, 256 and 88 rows
KINDS = {"stream": (3, 9000), "one": (12, 24000), "two": (45, 24000), "tiles": (150, 8000)}


def units_of_a_cta(torch, b, mask):
    """Of the tensor-memory kernel, on average: every (sequence, KV head, tile of 256 rows) has a cost of 3 besides."""
    group, places, units = b.q_heads // b.kv_heads, 0, 0
    for c, n in zip(b.ctx, b.nodes):
        for rt in range(-(-int(n) * group // 256)):
            end = int(c) + (int(n) if mask is not None else min(int(n), -(-(rt + 1) * 256 // group)))
            units += b.kv_heads * -(-end // 128)
            places += b.kv_heads * (-(-end // 128) + 3)
    return units / torch.cuda.get_device_properties(0).multi_processor_count


def entries(b, a, s, n):
    """Batch.entries of layer 0, a page at a time."""
    pages = a[0, b.table[s, :-(-n // b.page)]]      # [pages][kv_heads][page][dim]
    return np.ascontiguousarray(pages.transpose(0, 2, 1, 3)).reshape(-1, b.kv_heads, b.dim)[:n]


def attention(torch, b, q, mask, scale, seen=None):
    """_paged.attention (the same bounds, all rows of a KV head at a time) on the GPU in 64 bits.  seen: [rows][slots] of every
    sequence instead of what the batch says."""
    group, u = b.q_heads // b.kv_heads, _paged.HALF_STEP[b.dtype]
    out, bound = np.full((2, b.n_tok, b.q_heads, b.dim), np.nan)
    lse, lse_bound = np.full((2, b.n_tok, b.q_heads), np.nan)
    for s in range(len(b.ctx)):
        r0, r1, n = int(b.row_begin[s]), int(b.row_begin[s + 1]), int(b.ctx[s] + b.nodes[s])
        if r1 == r0:
            continue
        k, v = (on_gpu(torch, entries(b, a, s, n)).double() for a in (b.k, b.v))
        see = on_gpu(torch, b.sees(s, mask) if seen is None else seen[s])
        k, v = (torch.where(see.any(0)[:, None, None], a, 0.0) for a in (k, v))      # what no row sees may be anything
        for g in range(b.kv_heads):
            rows = on_gpu(torch, q[r0:r1, g * group:(g + 1) * group]).double()
            for i0 in range(0, r1 - r0, 16):
                part = rows[i0:i0 + 16].reshape(-1, b.dim)
                look = see[i0:i0 + 16].repeat_interleave(group, 0)
                x = torch.where(look, scale * (part @ k[:, g].T), -torch.inf)
                top = x.amax(1, keepdim=True).clamp_min(-1e300)
                p = torch.exp(x - top)
                total = p.sum(1, keepdim=True)
                share = p / torch.where(total > 0, total, 1.0)
                count = look.sum(1, keepdim=True)
                d_score = (b.dim + 4) * 2.0 ** -24 * scale * torch.where(look, part.abs() @ k[:, g].abs().T, 0.0).amax(1, keepdim=True) + \
                    torch.where(look, x.abs(), 0.0).amax(1, keepdim=True) * 2.0 ** -22
                rel = u + 2 * d_score + 2.0 ** -20 + count * 2.0 ** -24
                o = share @ v[:, g]
                z = torch.where(total > 0, top + torch.log(total), -torch.inf)
                at = (slice(r0 + i0, min(r0 + i0 + 16, r1)), slice(g * group, (g + 1) * group))
                shape = (at[0].stop - at[0].start, group)
                out[at] = o.view(*shape, b.dim).cpu().numpy()
                bound[at] = ((share @ v[:, g].abs()) * rel + o.abs() * rel).view(*shape, b.dim).cpu().numpy()
                lse[at] = z.view(shape).cpu().numpy()
                lse_bound[at] = (2 * d_score + 2.0 ** -20 + count * 2.0 ** -24 + z.abs() * 2.0 ** -22).view(shape).cpu().numpy()
    return out, lse, bound, lse_bound


def compare(b, got, want, final=None):
    out, lse = got
    ref, ref_lse, tol, lse_tol = want
    n, final = b.live, _paged.HALF_STEP[b.dtype] if final is None else final
    limit = tol[:n] * (1 + final) + np.abs(ref[:n]) * final + 2.0 ** -25
    diff = np.abs(out[:n] - ref[:n])
    assert np.all(diff <= limit), f"worst {np.nanmax(diff / limit):.2f} of the bound"
    empty = np.isneginf(ref_lse[:n])
    assert np.array_equal(np.isneginf(lse[:n]), empty) and np.all(out[:n][empty] == 0)
    assert np.all(np.abs(lse[:n][~empty] - ref_lse[:n][~empty]) <= lse_tol[:n][~empty])
    assert np.all(out[n:] == 7.0) and np.all(lse[n:] == 7.0)


def run(gpu, b, mask, q, pool_kv=None, times=1, status=None):
    """Output and log-sum-exp; of several runs, all with the same bits.  status: what the pool has to report."""
    torch, binding = gpu
    k, v, pool = pool_kv or cache_on_gpu(gpu, b)
    batch, dq = batch_on_gpu(gpu, b, mask=mask), on_gpu(torch, q).to(k.dtype)
    first = None
    for _ in range(times):
        out = torch.full(q.shape, 7.0, dtype=k.dtype, device="cuda")
        z = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
        pool.tree_attention(0, batch, dq, out, lse=z)
        if first is None:
            first = out, z
        assert torch.equal(out.view(torch.int16), first[0].view(torch.int16)) and torch.equal(z.view(torch.int32), first[1].view(torch.int32))
    if status:
        with pytest.raises(binding.PrimaError) as e:
            pool.sync()
        assert e.value.code == binding.ERR_DEVICE and status in str(e.value)
    else:
        pool.sync()
    return first[0].float().cpu().numpy(), first[1].cpu().numpy()


def peaks(b, slope):
    """Keys and queries whose scores are tents over the positions: `slope` binary exponents per 128 positions up to a peak,
    and down again behind it, at another place for every row.  Half of the rows of a warp rise while the others have their mass
    already; every eighth sees all positions alike."""
    dim, n = b.dim, int(b.ctx.max() + b.nodes.max())
    width = 5 * 128
    height = 5 * slope * np.log(2.0)
    j = np.arange(n)
    centre = (np.arange(dim) + 0.5) * n / dim
    tent = np.maximum(0.0, 1 - np.abs(j[:, None] - centre) / width) * (height / (4 * dim ** -0.5))
    for s in range(len(b.ctx)):
        for i in range(int(b.ctx[s] + b.nodes[s])):
            page, row = b.place(s, i)
            b.k[:, page, :, row] = _paged.rounded((0.05 * b.k[:, page, :, row] + tent[i]).astype(np.float32), b.dtype)
    q = 0.05 * b.rs.standard_normal((b.n_tok, b.q_heads, dim)).astype(np.float32)
    for t in range(b.n_tok):
        for h in range(b.q_heads):
            x = t * b.q_heads + h
            if x % 8:
                q[t, h, x * 29 % dim] += 4
    return _paged.rounded(q, b.dtype)


@pytest.mark.parametrize("dim,dtype", [(128, "float16"), (64, "bfloat16")])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tree", [True, False])
def test_references_that_move_in_every_unit(gpu, kind, dim, dtype, tree):
    torch, _ = gpu
    nodes, ctx = KINDS[kind]
    b = Batch(200 + dim, ctx=[ctx], nodes=[nodes], page=64, q_heads=16, kv_heads=4, dim=dim, dtype=dtype, pad=1)
    q = peaks(b, 12.0)
    mask = b.trees(3)[0] if tree else None
    if kind != "stream":
        assert units_of_a_cta(torch, b, mask) >= 3
    want = attention(torch, b, q, mask, dim ** -0.5)
    compare(b, run(gpu, b, mask, q, times=30), want)


@pytest.mark.parametrize("nodes", [10, 33])
def test_segments_that_follow_one_another(gpu, nodes):
    """Many segments of one unit per CTA: what the two warps of a row exchange at the end of one segment and at the beginning
    of the next lies in the same place.  Keys are large and sums small (one position has all of the weight), so that a maximum in
    the place of a sum shows."""
    torch, _ = gpu
    n = 300
    b = Batch(210, ctx=np.random.RandomState(1).randint(20, 128 - nodes, n), nodes=[nodes] * n, page=16, q_heads=16, kv_heads=4, dim=64)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 16, 64)).astype(np.float32) * 8, b.dtype)
    mask, _ = b.trees()
    assert units_of_a_cta(torch, b, mask) >= 8
    compare(b, run(gpu, b, mask, q, times=30), attention(torch, b, q, mask, 0.125))


@pytest.mark.parametrize("nodes,dim", [(10, 64), (10, 128), (40, 128)])
def test_first_segments_of_one_unit(gpu, nodes, dim):
    """A CTA's first segment has one unit and the next one's queries are ready at once: the copies do not wait for a state
    that has passed."""
    torch, _ = gpu
    n = 370
    b = Batch(220, ctx=[100 - nodes] * n, nodes=[nodes] * n, page=128, q_heads=8, kv_heads=2, dim=dim, dtype="bfloat16")
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 8, dim)).astype(np.float32), b.dtype)
    mask, _ = b.trees()
    compare(b, run(gpu, b, mask, q, times=50), attention(torch, b, q, mask, dim ** -0.5))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("nodes,page,pages,ctx", [(2, 8, 3, 25), (3, 8, 19, 1000), (12, 16, 10, 1000), (45, 16, 5, 100), (45, 16, 10, 150)])
def test_positions_beyond_the_table_are_not_seen(gpu, nodes, page, pages, ctx, tree, dim):
    """A sequence longer than its row of the table can name: its rows see what the table names, and the status says so."""
    torch, binding = gpu
    capacity = page * pages
    b = Batch(230, ctx=[ctx, capacity - nodes], nodes=[nodes, nodes], page=page, q_heads=8, kv_heads=2, dim=dim)
    mask = b.trees()[0] if tree else None
    seen = [b.sees(s, mask) for s in range(2)]
    seen[0][:, capacity:] = False
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 8, dim)).astype(np.float32), b.dtype)
    want = attention(torch, b, q, mask, dim ** -0.5, seen)
    b.table = np.ascontiguousarray(b.table[:, :pages])
    compare(b, run(gpu, b, mask, q, status="slot"), want)


@pytest.mark.parametrize("kind", KINDS)
def test_a_row_without_a_number_has_no_sum(gpu, kind):
    """NaN in a query: output and log-sum-exp of that row are NaN, not those of a row that sees nothing; other rows do not
    notice."""
    torch, _ = gpu
    nodes, ctx = KINDS[kind]
    for c in (ctx, 70):
        b = Batch(240, ctx=[c, 5], nodes=[nodes, nodes], page=64, q_heads=4, kv_heads=1, dim=64)
        mask, _ = b.trees(3)
        q = _paged.rounded(b.rs.standard_normal((b.n_tok, 4, 64)).astype(np.float32), b.dtype)
        want = attention(torch, b, q, mask, 0.125)
        bad = [(0, 1), (nodes - 1, 3), (nodes, 0)]
        for t, h in bad:
            q[t, h, 17] = np.nan
        out, lse = run(gpu, b, mask, q)
        for t, h in bad:
            assert np.all(np.isnan(out[t, h])) and np.isnan(lse[t, h])
            out[t, h], lse[t, h] = want[0][t, h], want[1][t, h]
        compare(b, (out, lse), want)


@pytest.mark.parametrize("gain", [1e-3, 12.0, 40.0])
@pytest.mark.parametrize("kind", KINDS)
def test_score_ranges_over_many_units(gpu, kind, gain):
    """From an even softmax to one where a single position takes all."""
    torch, _ = gpu
    nodes, ctx = KINDS[kind]
    b = Batch(250, ctx=[ctx], nodes=[nodes], page=32, q_heads=16, kv_heads=4, dim=64)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 16, 64)).astype(np.float32) * gain, b.dtype)
    mask = b.trees(3)[0]
    compare(b, run(gpu, b, mask, q, times=3), attention(torch, b, q, mask, 0.125))


@pytest.mark.parametrize("dim,dtype", [(128, "float16"), (64, "bfloat16")])
@pytest.mark.parametrize("junk", [np.inf, -np.inf, np.nan, 65504.0])
@pytest.mark.parametrize("kind", KINDS)
def test_stale_entries_do_no_harm_behind_many_units(gpu, kind, junk, dim, dtype):
    """Whatever no row sees (behind a sequence's end, on pages of nobody, a node that is seen by no row) may hold anything, and
    keys that a row does not see, too."""
    torch, _ = gpu
    nodes, ctx = KINDS[kind]
    b = Batch(260 + dim, ctx=[ctx, 3, 250], nodes=[nodes, nodes, nodes], page=16, q_heads=16, kv_heads=4, dim=dim, dtype=dtype, pad=1)
    mask, _ = b.trees(3)
    mask[nodes - 1, (nodes - 1) // 64] &= ~np.int64(np.uint64(1 << (nodes - 1) % 64).view(np.int64))      # the last node of the first sequence
    assert not b.sees(0, mask)[:, -1].any()
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 16, dim)).astype(np.float32), b.dtype)
    want = attention(torch, b, q, mask, dim ** -0.5)
    keep = np.zeros((b.n_pages, b.page), bool)
    for s in range(3):
        for j in range(int(b.ctx[s] + nodes) - (s == 0)):
            keep[b.place(s, j)] = True
    for a in (b.k, b.v):
        a[:] = np.where(keep[None, :, None, :, None], a, np.float32(junk))
    compare(b, run(gpu, b, mask, q), want)
    # a key that only its own row sees
    t = int(b.row_begin[2]) + 1
    mask[b.row_begin[2]:, 0] &= ~np.int64(2)
    mask[t, 0] |= 2
    want = attention(torch, b, q, mask, dim ** -0.5)
    page, row = b.place(2, 251)
    b.k[:, page, :, row] = junk
    out, lse = run(gpu, b, mask, q)
    out[t], lse[t] = want[0][t], want[1][t]
    compare(b, (out, lse), want)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [8, 64, 256])
@pytest.mark.parametrize("kind", KINDS)
def test_bad_pages_among_many_units(gpu, kind, page, dim):
    """Positions on pages that the pool does not have are not seen: at the beginning, in runs, alone, and at the end, under the
    rows of the step."""
    torch, _ = gpu
    nodes, ctx = KINDS[kind]
    b = Batch(270, ctx=[ctx, 700], nodes=[nodes, nodes], page=page, q_heads=16, kv_heads=4, dim=dim, dtype="bfloat16")
    mask, _ = b.trees(3)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 16, dim)).astype(np.float32), b.dtype)
    used = -(-(ctx + nodes) // page)
    lost = sorted({0, used // 3, used // 3 + 1, used // 3 + 2, used // 2, used - 1})
    seen = [b.sees(s, mask) for s in range(2)]
    for p in lost:
        seen[0][:, p * page:(p + 1) * page] = False
    want = attention(torch, b, q, mask, dim ** -0.5, seen)
    b.table[0, lost] = np.array([-1, b.n_pages, -2 ** 31, 2 ** 31 - 1, -7, b.n_pages + 5], np.int64)[:len(lost)].astype(np.int32)
    compare(b, run(gpu, b, mask, q, times=3, status="page id"), want)


@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_see_nothing_beside_others(gpu, kind):
    torch, _ = gpu
    nodes, ctx = KINDS[kind]
    b = Batch(280, ctx=[0, 0, ctx], nodes=[nodes, nodes, nodes], page=16, q_heads=16, kv_heads=4, dim=64, pad=2)
    mask, _ = b.trees(3)
    mask[:nodes] = 0                       # a whole sequence
    mask[[nodes, nodes + 2]] = 0           # rows beside others in their tile
    mask[b.row_begin[2] + 1] = 0           # sees its context only
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 16, 64)).astype(np.float32), b.dtype)
    want = attention(torch, b, q, mask, 0.125)
    assert np.all(np.isneginf(want[1][:nodes])) and np.isfinite(want[1][b.row_begin[2]:b.live]).all()
    compare(b, run(gpu, b, mask, q), want)


@pytest.mark.parametrize("kind", ["one", "two"])
def test_two_graphs_of_many_units_replayed_side_by_side(gpu, kind):
    """Captured calls with a workspace each, replayed at once on two streams with new lengths: many units, one, none."""
    torch, binding = gpu
    nodes, ctx = KINDS[kind]
    b = Batch(290, ctx=[ctx, 900], nodes=[nodes, nodes], page=64, q_heads=16, kv_heads=4, dim=64)
    mask, _ = b.trees(1)
    k, v, pool = cache_on_gpu(gpu, b)
    dev = on_gpu(torch, b.ctx)
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin), dev, b.n_tok, mask=on_gpu(torch, mask))
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 16, 64)).astype(np.float32), b.dtype)
    dq = on_gpu(torch, q).half()
    outs, lses, graphs = [torch.zeros_like(dq) for _ in range(2)], [torch.zeros(dq.shape[:2], device="cuda") for _ in range(2)], []
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pool.tree_attention(0, batch, dq, outs[i], lse=lses[i])
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for lens in ([ctx, 900], [40, 0], [5000, 127], [0, 0]):
        dev.copy_(torch.tensor(lens, dtype=torch.int32))
        b.ctx = np.array(lens, np.int32)
        torch.cuda.synchronize()
        for _ in range(5):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        pool.sync()
        want = attention(torch, b, q, mask, 0.125)
        for o, z in zip(outs, lses):
            compare(b, (o.float().cpu().numpy(), z.cpu().numpy()), want)
    del graphs


@pytest.mark.parametrize("exponent,dtype", [(12.0, "float16"), (20.0, "float16"), (24.3, "float16"), (25.3, "float16"), (28.0, "float16"), (25.3, "bfloat16")])
@pytest.mark.parametrize("kind", [*KINDS, "stream whole", "one whole", "two whole"])
def test_a_long_even_context_under_one_position_that_has_most(gpu, kind, exponent, dtype):
    """One position has a score so far above all others that each of them has a weight of 2^-exponent of its own; thousands of
    them count all the same, and must not be rounded away one by one.  "whole": so many sequences that most are not cut."""
    torch, _ = gpu
    nodes, ctx = KINDS[kind.split()[0]]
    n = 1
    if "whole" in kind:
        n, ctx = 80, 3000
    b = Batch(300, ctx=[ctx] * n, nodes=[nodes] * n, page=64, q_heads=16, kv_heads=4, dim=64, dtype=dtype)
    b.k[:] = 0
    b.v[:] = _paged.rounded(1 + 0.1 * b.v, dtype)
    for s in range(n):
        for j, size in ((5, exponent), (ctx // 2, exponent - 3), (ctx - 70, exponent)):
            page, row = b.place(s, j)
            b.k[:, page, :, row, 0] = _paged.rounded(np.array([size], np.float32), dtype)
            b.v[:, page, :, row] = 0
    q = np.zeros((b.n_tok, 16, 64), np.float32)
    q[:, :, 0] = _paged.rounded(np.array([8 * np.log(2.0)], np.float32), dtype)
    want = list(attention(torch, b, q, None, 0.125))
    # binary16: p is held as 2^7 and more times its share of the row's largest, so that half a step of its smallest numbers,
    # 2^-25, is 2^-32 of the largest: 2^(28 - 32), a sixteenth, of the weights here at most
    if dtype == "float16":
        for s in range(n):
            seen = np.abs(entries(b, b.v, s, ctx + nodes)).sum(0)      # [kv_heads][dim]
            want[2][b.row_begin[s]:b.row_begin[s + 1]] += 2.0 ** -32 * np.repeat(seen, 4, 0)
    assert np.nanmax(want[2] / want[0]) < 0.2
    compare(b, run(gpu, b, None, q), want)
