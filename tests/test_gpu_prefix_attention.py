"""Attention of batches behind shared prefixes, against softmax in 64 bits."""
import numpy as np
import pytest

from tests import _paged, _prefix
from tests._prefix import PrefixBatch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def prefix_on_gpu(gpu, b):
    torch, binding = gpu
    return binding.PrefixBatch(on_gpu(torch, b.prefix_table), on_gpu(torch, b.prefix), on_gpu(torch, b.groups))


def run(gpu, b, mask=None, layer=0, scale=None, out_dtype=None, q=None, pool_kv=None, lse=True):
    torch, binding = gpu
    k, v, pool = pool_kv or cache_on_gpu(gpu, b)
    if q is None:
        q = _paged.rounded(b.rs.standard_normal((b.n_tok, b.q_heads, b.dim)).astype(np.float32) * 1.5, b.dtype)
    out = torch.full(q.shape, 7.0, dtype=getattr(torch, out_dtype or b.dtype), device="cuda")
    z = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda") if lse else None
    pool.prefix_attention(layer, batch_on_gpu(gpu, b, mask=mask), prefix_on_gpu(gpu, b), on_gpu(torch, q).to(k.dtype), out, scale=scale, lse=z)
    pool.sync()
    return q, out.float().cpu().numpy(), z.cpu().numpy() if lse else None


def check(gpu, b, mask=None, layer=0, scale=None, out_dtype=None, q=None, pool_kv=None):
    q, out, lse = run(gpu, b, mask, layer, scale, out_dtype, q, pool_kv)
    want, want_lse, tol, lse_tol = _prefix.prefix_attention(b, layer, q, mask, scale or b.dim ** -0.5)
    n = b.live
    final = _paged.HALF_STEP[out_dtype or b.dtype]
    limit = tol[:n] * (1 + final) + np.abs(want[:n]) * final + 2.0 ** -25
    assert np.all(np.abs(out[:n] - want[:n]) <= limit), f"worst {np.nanmax(np.abs(out[:n] - want[:n]) / limit):.2f} of the bound"
    empty = np.isneginf(want_lse[:n])
    assert np.array_equal(np.isneginf(lse[:n]), empty) and np.all(out[:n][empty] == 0)
    assert np.all(np.abs(lse[:n][~empty] - want_lse[:n][~empty]) <= lse_tol[:n][~empty])
    assert np.all(out[n:] == 7.0) and np.all(lse[n:] == 7.0)      # rows behind the last sequence
    return out


SHAPES = [  # ctx, nodes, prefix, groups, page, q_heads, kv_heads, dim
    ([0], [1], [1], [0, 1], 16, 1, 1, 128), ([3, 9], [1, 1], [127], [0, 2], 16, 4, 1, 128), ([0, 0, 7], [1, 1, 1], [128], [0, 3], 8, 6, 2, 64),
    ([5, 60], [1, 2], [129], [0, 2], 64, 8, 2, 128), ([200, 1, 0], [3, 1, 5], [700], [0, 3], 32, 5, 1, 128), ([10] * 30, [1] * 30, [300], [0, 30], 16, 8, 1, 128),
    ([10] * 33, [1] * 33, [1000], [0, 33], 16, 8, 1, 64), ([1, 2, 3, 140, 5], [1, 40, 2, 9, 1], [257], [0, 5], 128, 6, 1, 128),
    ([5, 0, 130, 64, 90, 1], [3, 1, 0, 16, 7, 40], [50, 0, 400], [0, 2, 3, 6], 16, 6, 2, 128), ([5, 9, 8, 7], [1, 2, 3, 4], [90], [1, 3], 16, 4, 2, 64),
    ([4, 5, 6], [2, 2, 2], [33, 65], [0, 0, 3], 16, 4, 4, 128), ([0, 0], [300, 2], [500], [0, 2], 16, 2, 1, 64),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"case{i}" for i in range(len(SHAPES))])
@pytest.mark.parametrize("kind", ["tree", "causal"])
def test_shapes(gpu, dtype, shape, kind):
    ctx, nodes, prefix, groups, page, H, G, D = shape
    b = PrefixBatch(600, ctx, nodes, prefix, groups, page, q_heads=H, kv_heads=G, dim=D, dtype=dtype, pad=2)
    check(gpu, b, b.trees(words=5)[0] if kind == "tree" else None)


@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 16, 64])
def test_heads_sharing_a_kv_head(gpu, group):
    b = PrefixBatch(601, [20, 33, 4], [2, 3, 1], [400], [0, 3], 16, q_heads=2 * group, kv_heads=2, dim=64)
    check(gpu, b)


@pytest.mark.parametrize("length", [0, 1, 127, 128, 129, 1025, 5000])
def test_lengths_of_the_prefix(gpu, length):
    b = PrefixBatch(602, [2, 0, 9], [1, 1, 1], [length], [0, 3], 8, q_heads=4, kv_heads=2, dim=128, dtype="bfloat16")
    check(gpu, b)


def test_it_is_tree_attention_with_the_prefix_in_every_table(gpu):
    """The same rows over caches that hold the prefix in front of their own positions (whole pages of it)."""
    torch, binding = gpu
    b = PrefixBatch(603, [5, 17, 30], [2, 1, 4], [96], [0, 3], 16, q_heads=8, kv_heads=2, dim=128)
    kv = cache_on_gpu(gpu, b)
    q, out, lse = run(gpu, b, pool_kv=kv)
    table = np.concatenate([np.repeat(b.prefix_table[:, :6], 3, 0), b.table], 1)
    batch = binding.PagedBatch(on_gpu(torch, table), on_gpu(torch, b.row_begin), on_gpu(torch, b.ctx + 96), b.n_tok)
    want, z = torch.empty(q.shape, dtype=torch.float16, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    kv[2].tree_attention(0, batch, on_gpu(torch, q).half(), want, lse=z)
    kv[2].sync()
    # probabilities and results of both are rounded by half a step each: 2^-11 of values of at most |v|
    assert np.abs(out - want.float().cpu().numpy()).max() <= 4 * 2.0 ** -11 * np.abs(b.v).max()
    assert np.abs(lse - z.cpu().numpy()).max() <= 2.0 ** -18


def test_rows_that_see_nothing_of_their_own(gpu):
    """Behind a prefix they see that; without one, nothing: zeros and -infinity."""
    b = PrefixBatch(604, [0, 0, 0, 6], [3, 2, 2, 1], [40], [1, 3], 16, q_heads=4, kv_heads=2, dim=64)
    mask = np.zeros((b.n_tok, 1), np.int64)
    mask[0] = 1
    out = check(gpu, b, mask)
    assert np.all(out[1:3] == 0) and np.any(out[3:7] != 0)


@pytest.mark.parametrize("junk", [np.inf, np.nan, 65504.0])
def test_stale_entries_do_no_harm(gpu, junk):
    """Behind the end of a prefix, on spare pages and in slots that no row has, the cache holds anything."""
    b = PrefixBatch(605, [4, 70, 0], [1, 2, 5], [201], [0, 3], 16, q_heads=6, kv_heads=2, dim=128)
    live = np.zeros(b.k.shape[:4], bool)
    for s in range(3):
        for j in range(int(b.ctx[s] + b.nodes[s])):
            p, r = b.place(s, j)
            live[:, p, :, r] = True
    for j in range(201):
        live[:, b.prefix_table[0, j // 16], :, j % 16] = True
    b.k[~live] = junk
    b.v[~live] = junk
    check(gpu, b)


@pytest.mark.parametrize("gain", [1e-3, 1.0, 12.0, 40.0])
def test_score_ranges(gpu, gain):
    b = PrefixBatch(606, [40, 3, 0, 9] * 5, [1, 2, 1, 1] * 5, [300], [0, 20], 16, q_heads=8, kv_heads=1, dim=128)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 8, 128)).astype(np.float32) * gain, "float16")
    check(gpu, b, q=q)


def test_prefix_and_own_positions_of_very_different_weight(gpu):
    """Scores that rise along the prefix, and own positions far above or below all of it."""
    for own in (0.2, -3.0, 3.0):
        b = PrefixBatch(607, [30, 2], [2, 1], [640], [0, 2], 16, q_heads=2, kv_heads=1, dim=64)
        q = np.ones((b.n_tok, 2, 64), np.float32)
        for j in range(640):
            b.k[:, b.prefix_table[0, j // 16], :, j % 16] = _paged.rounded(np.float32(j / 300 - 1) + 0 * b.k[0, 0, 0, 0], "float16")
        for s in range(2):
            for j in range(int(b.ctx[s] + b.nodes[s])):
                p, r = b.place(s, j)
                b.k[:, p, :, r] = own
        check(gpu, b, q=q, scale=1.0)


def test_scale_layer_output_type_and_no_lse(gpu):
    b = PrefixBatch(608, [30, 2], [2, 1], [140], [0, 2], 16, layers=3, q_heads=2, kv_heads=1, dim=64, dtype="bfloat16")
    a = check(gpu, b, layer=2, scale=0.3, out_dtype="float32")
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 2, 64)).astype(np.float32), "bfloat16")
    with_lse, without = run(gpu, b, q=q)[1], run(gpu, b, q=q, lse=False)[1]
    assert np.array_equal(with_lse, without) and a.shape == with_lse.shape


def test_many_sequences_and_many_prefixes(gpu):
    rs = np.random.RandomState(5)
    groups = np.sort(np.concatenate([[0, 300], rs.randint(0, 301, 39)]))
    b = PrefixBatch(609, rs.randint(0, 20, 300), rs.randint(0, 3, 300), rs.randint(0, 200, 40), groups, 8, q_heads=2, kv_heads=1, dim=64, pad=1)
    check(gpu, b)


@pytest.mark.parametrize("rows", [255, 256, 257, 600])
def test_tiles_of_rows(gpu, rows):
    b = PrefixBatch(610, [3, 5], [rows - 1, 1], [400], [0, 2], 32, q_heads=1, kv_heads=1, dim=128)
    check(gpu, b)


def test_positions_on_bad_pages_are_not_seen(gpu):
    torch, binding = gpu
    b = PrefixBatch(611, [20, 9], [1, 2], [300], [0, 2], 16, q_heads=4, kv_heads=1, dim=64)
    kv = cache_on_gpu(gpu, b)
    table, own = b.prefix_table.copy(), b.table.copy()
    table[0, 3], table[0, 10], own[0, 0] = -1, b.n_pages, 1 << 30
    prefix = binding.PrefixBatch(on_gpu(torch, table), on_gpu(torch, b.prefix), on_gpu(torch, b.groups))
    batch = binding.PagedBatch(on_gpu(torch, own), on_gpu(torch, b.row_begin), on_gpu(torch, b.ctx), b.n_tok)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 4, 64)).astype(np.float32), "float16")
    out, lse = torch.empty(q.shape, dtype=torch.float16, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    kv[2].prefix_attention(0, batch, prefix, on_gpu(torch, q).half(), out, lse=lse)
    with pytest.raises(binding.PrimaError) as e:
        kv[2].sync()
    assert "page" in str(e.value)
    # the definition over what is left
    gone = {3 * 16 + i for i in range(16)} | {10 * 16 + i for i in range(16)}
    at = [j for j in range(300) if j not in gone]
    for s in range(2):
        for i in range(int(b.nodes[s])):
            t = int(b.row_begin[s]) + i
            mine = [j for j in range(int(b.ctx[s]) + i + 1) if not (s == 0 and j < 16)]
            k, v = (np.concatenate([b.prefix_entries(a, 0, 0)[at], np.array([a[0, own[s, j // 16], :, j % 16] for j in mine]).reshape(-1, 1, 64)]).astype(np.float64) for a in (b.k, b.v))
            x = np.einsum("hd,ld->hl", q[t].astype(np.float64), k[:, 0]) / 8
            p = np.exp(x - x.max(-1, keepdims=True))
            want = (p / p.sum(-1, keepdims=True)) @ v[:, 0]
            assert np.abs(out[t].float().cpu().numpy() - want).max() <= 4 * 2.0 ** -11 * np.abs(b.v).max()
            assert np.abs(lse[t].cpu().numpy() - np.log(np.exp(x).sum(-1))).max() <= 2.0 ** -16


def test_bad_prefixes_count_as_none(gpu):
    torch, binding = gpu
    b = PrefixBatch(612, [20, 9, 5], [1, 2, 1], [50, 60], [0, 2, 3], 16, q_heads=4, kv_heads=1, dim=64)
    kv = cache_on_gpu(gpu, b)
    q, batch = _paged.rounded(b.rs.standard_normal((b.n_tok, 4, 64)).astype(np.float32), "float16"), batch_on_gpu(gpu, b)

    def call(length, groups):
        out = torch.empty(q.shape, dtype=torch.float16, device="cuda")
        kv[2].prefix_attention(0, batch, binding.PrefixBatch(on_gpu(torch, b.prefix_table), on_gpu(torch, np.array(length, np.int32)), on_gpu(torch, np.array(groups, np.int32))),
                               on_gpu(torch, q).half(), out)
        return out
    def near(x, y):      # other lengths cut the work elsewhere: two roundings of each
        return (x.float() - y.float()).abs().max().item() <= 4 * 2.0 ** -11 * np.abs(b.v).max()
    none, right = call([0, 0], [0, 2, 3]), call([50, 60], [0, 2, 3])
    kv[2].sync()
    assert not near(none[:3], right[:3]) and not near(none[3:], right[3:])
    for length, groups, want in (([-1, 60], [0, 2, 3], 3), ([50, 60], [-1, 2, 3], 3), ([50, 60], [0, 2, 4], 0)):
        got = call(length, groups)
        with pytest.raises(binding.PrimaError):
            kv[2].sync()
        first = none if want == 3 else right
        second = right if want == 3 else none
        assert near(got[:3], first[:3]) and near(got[3:], second[3:])
    # positions behind the table
    got = call([50, 10 ** 6], [0, 2, 3])
    with pytest.raises(binding.PrimaError) as e:
        kv[2].sync()
    assert "slot" in str(e.value) and near(got[:3], right[:3])


def test_runs_give_the_same_bits_and_two_streams_do_not_meet(gpu):
    torch, binding = gpu
    b = PrefixBatch(613, [40, 300, 5, 60] * 4, [1, 2, 3, 1] * 4, [2000], [0, 16], 16, q_heads=8, kv_heads=2, dim=128)
    kv = cache_on_gpu(gpu, b)
    batch, prefix = batch_on_gpu(gpu, b), prefix_on_gpu(gpu, b)
    q = [torch.randn((b.n_tok, 8, 128), device="cuda").half() for _ in range(2)]
    out = [torch.empty_like(x) for x in q]
    want = []
    for i in range(2):
        kv[2].prefix_attention(0, batch, prefix, q[i], out[i])
        want.append(out[i].clone())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            out[i].zero_()
        torch.cuda.synchronize()
        for i in range(2):
            kv[2].prefix_attention(0, batch, prefix, q[i], out[i], stream=streams[i])
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    kv[2].sync()


def test_two_graphs_replayed_with_new_lengths(gpu):
    """Lengths, prefixes and tables are read when the graph runs."""
    torch, binding = gpu
    b = PrefixBatch(614, [40, 200, 5], [1, 2, 3], [900, 300], [0, 2, 3], 16, q_heads=8, kv_heads=2, dim=64)
    kv = cache_on_gpu(gpu, b)
    ctx, length = on_gpu(torch, b.ctx), on_gpu(torch, b.prefix)
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin), ctx, b.n_tok)
    prefix = binding.PrefixBatch(on_gpu(torch, b.prefix_table), length, on_gpu(torch, b.groups))
    q = torch.randn((b.n_tok, 8, 64), device="cuda").half()
    outs, graphs = [torch.empty_like(q) for _ in range(2)], []
    kv[2].prefix_attention(0, batch, prefix, q, outs[0])
    torch.cuda.synchronize()
    for out in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kv[2].prefix_attention(0, batch, prefix, q, out)
        graphs.append(g)
    for own, shared in (([40, 200, 5], [900, 300]), ([0, 3, 1], [1, 0]), ([7, 100, 2], [640, 299])):
        ctx.copy_(torch.tensor(own, dtype=torch.int32))
        length.copy_(torch.tensor(shared, dtype=torch.int32))
        want = torch.empty_like(q)
        kv[2].prefix_attention(0, batch, prefix, q, want)
        for out in outs:
            out.zero_()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    kv[2].sync()


def test_argument_errors(gpu):
    torch, binding = gpu
    b = PrefixBatch(615, [4], [2], [20], [0, 1], 16, q_heads=4, kv_heads=2, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    batch, prefix = batch_on_gpu(gpu, b), prefix_on_gpu(gpu, b)
    q = torch.zeros((2, 4, 64), dtype=torch.float16, device="cuda")
    out = torch.empty_like(q)
    pool.prefix_attention(0, batch, prefix, q, out)
    for kw in (dict(layer=1), dict(layer=-1), dict(scale=0.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(out=torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")),
               dict(q=q[:, :3].contiguous(), out=out[:, :3].contiguous()), dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))):
        args = {"layer": 0, "q": q, "out": out, **kw}
        layer, qq, oo = args.pop("layer"), args.pop("q"), args.pop("out")
        with pytest.raises(binding.PrimaError) as e:
            pool.prefix_attention(layer, batch, prefix, qq, oo, **args)
        assert e.value.code == binding.ERR_ARG
    for qq, oo in ((q.float(), out), (q[:1], out), (q, out[:1])):
        with pytest.raises(ValueError):
            pool.prefix_attention(0, batch, prefix, qq, oo)
    i32 = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in ((i32, i32[:1], i32[:2]), (i32.view(1, 4), i32[:1], i32[:3]), (i32.view(1, 4), i32[:1].float(), i32[:2]), (i32.view(1, 4).cpu(), i32[:1], i32[:2])):
        with pytest.raises(ValueError):
            binding.PrefixBatch(*bad)
    pool.sync()
