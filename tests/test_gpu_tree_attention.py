"""Attention of trees, chains and single tokens over the paged cache, against softmax in 64 bits."""
import numpy as np
import pytest

from tests import _paged
from tests._paged import Batch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def run(gpu, b, mask, layer=0, scale=None, out_dtype=None, q=None, pool_kv=None, lse=True):
    torch, binding = gpu
    k, v, pool = pool_kv or cache_on_gpu(gpu, b)
    if q is None:
        q = _paged.rounded(b.rs.standard_normal((b.n_tok, b.q_heads, b.dim)).astype(np.float32) * 1.5, b.dtype)
    out = torch.full(q.shape, 7.0, dtype=getattr(torch, out_dtype or b.dtype), device="cuda")
    z = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda") if lse else None
    pool.tree_attention(layer, batch_on_gpu(gpu, b, mask=mask), on_gpu(torch, q).to(k.dtype), out, scale=scale, lse=z)
    pool.sync()
    return q, out.float().cpu().numpy(), z.cpu().numpy() if lse else None


def check(gpu, b, mask, layer=0, scale=None, out_dtype=None, q=None, pool_kv=None):
    q, out, lse = run(gpu, b, mask, layer, scale, out_dtype, q, pool_kv)
    want, want_lse, tol, lse_tol = _paged.attention(b, layer, q, mask, scale or b.dim ** -0.5)
    n = b.live
    final = _paged.HALF_STEP[out_dtype or b.dtype]
    worst = np.abs(out[:n] - want[:n]) / (tol[:n] + np.abs(want[:n]) * final + 1e-30 + 2.0 ** -25)
    assert np.all(np.abs(out[:n] - want[:n]) <= tol[:n] * (1 + final) + np.abs(want[:n]) * final + 2.0 ** -25), f"worst {np.nanmax(worst):.2f} of the bound"
    empty = np.isneginf(want_lse[:n])
    assert np.array_equal(np.isneginf(lse[:n]), empty) and np.all(out[:n][empty] == 0)
    assert np.all(np.abs(lse[:n][~empty] - want_lse[:n][~empty]) <= lse_tol[:n][~empty])
    assert np.all(out[n:] == 7.0) and np.all(lse[n:] == 7.0)      # rows behind the last sequence
    return out


SHAPES = [  # ctx, nodes, page, q_heads, kv_heads, dim
    ([0], [1], 16, 1, 1, 128), ([1], [1], 8, 2, 1, 64), ([127], [1], 16, 8, 1, 128), ([128], [1], 16, 5, 1, 128), ([129], [2], 64, 8, 2, 64),
    ([300], [5], 16, 4, 2, 128), ([255], [16], 32, 8, 1, 128), ([1000], [17], 16, 8, 1, 128), ([700], [33], 128, 7, 1, 64), ([511], [64], 256, 8, 1, 128),
    ([5, 0, 130, 64, 900, 1], [3, 1, 0, 16, 7, 40], 16, 6, 2, 128), ([100, 4, 31], [1, 1, 1], 32, 4, 4, 64),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"case{i}" for i in range(len(SHAPES))])
@pytest.mark.parametrize("kind", ["tree", "causal"])
def test_shapes(gpu, dtype, shape, kind):
    ctx, nodes, page, H, G, D = shape
    b = Batch(100, ctx=ctx, nodes=nodes, page=page, q_heads=H, kv_heads=G, dim=D, dtype=dtype, pad=2)
    check(gpu, b, b.trees()[0] if kind == "tree" else None)


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 64])
def test_heads_sharing_a_kv_head(gpu, group):
    b = Batch(101, ctx=[200, 33], nodes=[6, 3], page=16, q_heads=2 * group, kv_heads=2, dim=64)
    check(gpu, b, b.trees()[0])


def test_a_tree_equals_its_branches_as_chains(gpu):
    """Every branch of a tree, run as a chain of its own, gives the row of the tree that ends it."""
    b = Batch(102, ctx=[77], nodes=[12], page=16, q_heads=4, kv_heads=2, dim=64)
    mask, _ = b.trees()
    q, out, _ = run(gpu, b, mask)
    for i in range(12):
        path = [a for a in range(12) if int(mask[i, 0]) >> a & 1]
        c = Batch(102, ctx=[77], nodes=[len(path)], page=16, q_heads=4, kv_heads=2, dim=64)
        c.k, c.v, c.table, c.n_pages = b.k.copy(), b.v.copy(), b.table, b.n_pages
        for j, a in enumerate(path):
            (pf, rf), (pt, rt) = b.place(0, 77 + a), b.place(0, 77 + j)
            c.k[:, pt, :, rt], c.v[:, pt, :, rt] = b.k[:, pf, :, rf], b.v[:, pf, :, rf]
        _, got, _ = run(gpu, c, None, q=q[path])
        assert np.abs(got[-1] - out[i]).max() <= 4 * 2.0 ** -11 * np.abs(b.v).max()      # two roundings of each


@pytest.mark.parametrize("words,n", [(1, 64), (2, 100), (4, 256), (1, 70)])
def test_wide_trees(gpu, words, n):
    """Several words of bits; nodes beyond the words are seen by none (not even by themselves)."""
    b = Batch(103, ctx=[65], nodes=[n], page=32, q_heads=2, kv_heads=1, dim=64, dtype="bfloat16")
    check(gpu, b, b.trees(words)[0])


def test_long_chains_need_no_mask(gpu):
    check(gpu, Batch(104, ctx=[0, 40], nodes=[300, 129], page=16, q_heads=2, kv_heads=1, dim=64), None)


def test_rows_that_see_nothing(gpu):
    b = Batch(105, ctx=[0, 0, 50], nodes=[3, 1, 2], page=16, q_heads=4, kv_heads=2, dim=128, dtype="bfloat16")
    mask, _ = b.trees()
    mask[0] = mask[2] = mask[3] = 0      # nothing in the context either
    mask[4] = 0                          # sees its context only
    check(gpu, b, mask)


def test_bits_beyond_the_sequence_are_ignored(gpu):
    b = Batch(106, ctx=[30, 7], nodes=[5, 5], page=16, q_heads=4, kv_heads=2, dim=64)
    mask, _ = b.trees()
    want = run(gpu, b, mask, q=np.ones((10, 4, 64), np.float32))[1]
    got = run(gpu, b, mask | np.int64(-32), q=np.ones((10, 4, 64), np.float32))[1]
    assert np.array_equal(want, got)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("junk", [np.inf, -np.inf, np.nan, 65504.0])
def test_stale_entries_do_no_harm(gpu, dtype, junk):
    """Entries behind a sequence's end, on the rest of its last page and on pages of nobody, hold anything; keys that a row does not see, too."""
    torch, binding = gpu
    b = Batch(107, ctx=[130, 3, 250], nodes=[4, 2, 6], page=16, q_heads=4, kv_heads=2, dim=64, dtype=dtype)
    mask, _ = b.trees()
    keep = np.zeros((b.n_pages, b.page), bool)
    for s in range(3):
        for j in range(int(b.ctx[s] + b.nodes[s])):
            keep[b.place(s, j)] = True
    # the last node of the first sequence is seen by no row at all
    mask[3] &= ~np.int64(1 << 3)
    for i in range(4):
        assert not int(mask[i, 0]) >> 3 & 1
    keep[b.place(0, 133)] = False
    for a in (b.k, b.v):
        a[:] = np.where(keep[None, :, None, :, None], a, np.float32(junk))
    clean = Batch(107, ctx=[130, 3, 250], nodes=[4, 2, 6], page=16, q_heads=4, kv_heads=2, dim=64, dtype=dtype)
    q, out, lse = run(gpu, b, mask)
    want, want_lse, tol, _ = _paged.attention(clean, 0, q, mask, 0.125)
    assert np.all(np.abs(out - want) <= tol * 1.01 + np.abs(want) * _paged.HALF_STEP[dtype] + 2.0 ** -25)
    # a key that only other rows see
    b.k[:, b.place(2, 255)[0], :, b.place(2, 255)[1]] = junk
    mask[:, 0] &= ~np.int64(1 << 5)
    mask[b.live - 1, 0] |= 1 << 5
    q2, out2, _ = run(gpu, b, mask, q=q)
    want, _, tol, _ = _paged.attention(clean, 0, q, mask, 0.125)
    n = b.live - 1
    assert np.all(np.abs(out2[:n] - want[:n]) <= tol[:n] * 1.01 + np.abs(want[:n]) * _paged.HALF_STEP[dtype] + 2.0 ** -25)


@pytest.mark.parametrize("gain", [1e-3, 1.0, 12.0, 40.0])
def test_score_ranges(gpu, gain):
    """From an even softmax to one where a single position takes all; far negative scores vanish."""
    b = Batch(108, ctx=[700], nodes=[5], page=32, q_heads=4, kv_heads=1, dim=128)
    q = _paged.rounded(b.rs.standard_normal((5, 4, 128)).astype(np.float32) * gain, b.dtype)
    check(gpu, b, b.trees()[0], q=q)


def test_scores_that_rise_along_the_context(gpu):
    """The running maximum moves at every tile, upwards and downwards."""
    for sign in (1, -1):
        b = Batch(109, ctx=[900], nodes=[3], page=16, q_heads=4, kv_heads=1, dim=64)
        for j in range(900):
            page, row = b.place(0, j)
            b.k[:, page, :, row] = _paged.rounded(np.full((1, 1, 64), sign * (j - 450) / 150.0, np.float32) + 0.1 * b.k[:, page, :, row], b.dtype)
        q = _paged.rounded(1 + 0.2 * b.rs.standard_normal((3, 4, 64)).astype(np.float32), b.dtype)
        check(gpu, b, b.trees()[0], q=q)


def test_scale_layer_output_type_and_no_lse(gpu):
    b = Batch(110, ctx=[100, 3], nodes=[4, 6], page=16, q_heads=6, kv_heads=3, dim=64, layers=3, dtype="bfloat16")
    mask, _ = b.trees()
    for layer in (0, 2):
        check(gpu, b, mask, layer=layer, scale=0.3, out_dtype="float32")
    q, out, _ = run(gpu, b, mask, q=np.ones((10, 6, 64), np.float32))
    _, again, _ = run(gpu, b, mask, q=np.ones((10, 6, 64), np.float32), lse=False)
    assert np.array_equal(out, again)


def test_many_sequences_of_one_token(gpu):
    rs = np.random.RandomState(3)
    n = 333
    check(gpu, Batch(111, ctx=rs.randint(0, 90, n), nodes=rs.randint(0, 2, n), page=16, q_heads=2, kv_heads=1, dim=64, pad=1), None)


def test_positions_on_bad_pages_are_not_seen(gpu):
    torch, binding = gpu
    b = Batch(112, ctx=[60, 20], nodes=[2, 2], page=16, q_heads=2, kv_heads=1, dim=64)
    want = check(gpu, b, None, q=np.ones((4, 2, 64), np.float32))
    k, v, pool = cache_on_gpu(gpu, b)
    for bad in (-1, b.n_pages, -2 ** 31, 2 ** 31 - 1):
        table = b.table.copy()
        table[0, 1] = bad
        out = torch.zeros((4, 2, 64), dtype=k.dtype, device="cuda")
        batch = binding.PagedBatch(on_gpu(torch, table), on_gpu(torch, b.row_begin), on_gpu(torch, b.ctx), 4)
        pool.tree_attention(0, batch, torch.ones((4, 2, 64), dtype=k.dtype, device="cuda"), out)
        with pytest.raises(binding.PrimaError) as e:
            pool.sync()
        assert e.value.code == binding.ERR_DEVICE and "page id" in str(e.value)
        got = out.float().cpu().numpy()
        assert np.array_equal(got[2:], want[2:]) and np.all(np.isfinite(got))
        kk, vv = (np.concatenate([b.entries(a, 0, 0, 62)[:16], b.entries(a, 0, 0, 62)[32:62]]) for a in (b.k, b.v))
        for i in range(2):
            x = kk[:, 0].astype(np.float64).sum(-1) * 0.125
            x[-1] = -np.inf if i == 0 else x[-1]
            p = np.exp(x - x.max())
            assert np.abs(got[i, 0] - (p / p.sum()) @ vv[:, 0]).max() < 0.01
    ctx = on_gpu(torch, np.array([60, 1 << 20], np.int32))      # beyond the table
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin), ctx, 4)
    pool.tree_attention(0, batch, torch.ones((4, 2, 64), dtype=k.dtype, device="cuda"), out)
    with pytest.raises(binding.PrimaError) as e:
        pool.sync()
    assert "slot" in str(e.value)
    assert np.array_equal(out.float().cpu().numpy()[:2], want[:2])


def test_runs_give_the_same_bits_and_two_streams_do_not_meet(gpu):
    torch, binding = gpu
    b = Batch(113, ctx=[3000, 200, 17], nodes=[20, 5, 1], page=16, q_heads=8, kv_heads=2, dim=128, dtype="bfloat16")
    mask, _ = b.trees()
    kv = cache_on_gpu(gpu, b)
    batch = batch_on_gpu(gpu, b, mask=mask)
    q = [torch.randn((26, 8, 128), device="cuda").bfloat16() for _ in range(2)]
    out = [torch.zeros_like(x) for x in q]
    want = []
    for i in range(2):
        kv[2].tree_attention(0, batch, q[i], out[i])
        want.append(out[i].clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(20):
        for i in range(2):
            kv[2].tree_attention(0, batch, q[i], out[i], stream=streams[i])
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_two_graphs_replayed_with_new_lengths(gpu):
    torch, binding = gpu
    b = Batch(114, ctx=[300, 50], nodes=[4, 4], page=16, q_heads=4, kv_heads=1, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    ctx = on_gpu(torch, b.ctx)
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin), ctx, 8)
    q = _paged.rounded(b.rs.standard_normal((8, 4, 64)).astype(np.float32), b.dtype)
    dq = on_gpu(torch, q).half()
    outs, graphs = [torch.zeros_like(dq) for _ in range(2)], []
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pool.tree_attention(0, batch, dq, outs[i])
        graphs.append(g)
    for lens in ([300, 50], [10, 51], [0, 0]):
        ctx.copy_(torch.tensor(lens, dtype=torch.int32))
        b.ctx = np.array(lens, np.int32)
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want, _, tol, _ = _paged.attention(b, 0, q, None, 0.125)
        for o in outs:
            got = o.float().cpu().numpy()
            assert np.all(np.abs(got - want) <= tol * 1.01 + np.abs(want) * 2.0 ** -11 + 2.0 ** -25)
    del graphs


def test_argument_errors(gpu):
    torch, binding = gpu
    b = Batch(115, ctx=[4], nodes=[2], page=8, dim=64, q_heads=4, kv_heads=2)
    k, v, pool = cache_on_gpu(gpu, b)
    batch = batch_on_gpu(gpu, b)
    q = torch.zeros((2, 4, 64), dtype=k.dtype, device="cuda")
    out = torch.zeros_like(q)
    odd = torch.zeros(2 * 4 * 64 + 1, dtype=k.dtype, device="cuda")[1:].view(2, 4, 64)
    ws = pool.tree_attention_workspace(batch)
    for call in (lambda: pool.tree_attention(1, batch, q, out), lambda: pool.tree_attention(0, batch, q.float(), out), lambda: pool.tree_attention(0, batch, q, out.bfloat16()),
                 lambda: pool.tree_attention(0, batch, q[:, :3].contiguous(), out[:, :3].contiguous()), lambda: pool.tree_attention(0, batch, q, out, scale=0.0),
                 lambda: pool.tree_attention(0, batch, q, out, scale=float("nan")), lambda: pool.tree_attention(0, batch, q, out, scale=-1.0),
                 lambda: pool.tree_attention(0, batch, q[:1], out), lambda: pool.tree_attention(0, batch, q, out, lse=torch.zeros((2, 4), device="cuda").half()),
                 lambda: pool.tree_attention(0, batch, odd, out), lambda: pool.tree_attention(0, batch, q, odd),
                 lambda: pool.tree_attention(0, batch, q, out, workspace=ws[:255]), lambda: pool.tree_attention(0, batch, q, out, workspace=ws[1:]),
                 lambda: batch_on_gpu(gpu, b, mask=np.zeros((2, 17), np.int64)) and pool.tree_attention(0, batch_on_gpu(gpu, b, mask=np.zeros((2, 17), np.int64)), q, out),
                 lambda: batch_on_gpu(gpu, b, mask=np.zeros((3, 1), np.int64))):
        with pytest.raises((ValueError, binding.PrimaError)):
            call()
