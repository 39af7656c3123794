"""The attention weight that cached positions receive, against sums in 64 bits."""
import numpy as np
import pytest

from tests import _paged, _prefix
from tests._paged import Batch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def inputs(b, spare=3, gain=1.5):
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, b.q_heads, b.dim)).astype(np.float32) * gain, b.dtype)
    slots = int((b.ctx + b.nodes).max()) + spare
    w = np.exp(b.rs.standard_normal((len(b.ctx), b.kv_heads, slots)) * 2).astype(np.float32)
    return q, w


def lse_of(b, layer, q, mask, scale):
    """As an attention leaves it: rounded to 32 bits; rows of padding hold anything."""
    z = _paged.attention(b, layer, q, mask, scale)[1]
    return np.where(np.isnan(z), 3.0, z).astype(np.float32)


def check(gpu, b, mask=None, layer=0, scale=None, decay=1.0, first_time=False, in_place=False, pos=None, q=None, lse=None, kv=None):
    torch, binding = gpu
    k, v, pool = kv or cache_on_gpu(gpu, b)
    given, w = inputs(b)
    q = given if q is None else q
    scale = scale or b.dim ** -0.5
    lse = lse_of(b, layer, q, mask, scale) if lse is None else lse
    dw = on_gpu(torch, w)
    out = dw if in_place else torch.full_like(dw, 9.0)
    born = torch.full(w.shape, -7, dtype=torch.int32, device="cuda")
    pool.attention_weights(layer, batch_on_gpu(gpu, b, pos, mask), on_gpu(torch, q).to(k.dtype), on_gpu(torch, lse), out, weight_in=None if first_time else dw, decay=decay, born=born,
                           scale=scale)
    pool.sync()
    want, bound = _prefix.weights(b, layer, q, lse, mask, scale, None if first_time else w, np.float32(decay))
    got, at = out.cpu().numpy(), born.cpu().numpy()
    for s in range(len(b.ctx)):
        n, c = (int(b.ctx[s] + b.nodes[s]) if b.nodes[s] else 0), int(b.ctx[s])
        err = np.abs(got[s, :, :n] - want[s, :, :n])
        assert np.all(err <= bound[s, :, :n] + 2.0 ** -126), f"worst {np.nanmax(err / (bound[s, :, :n] + 1e-38)):.2f} of the bound"
        assert np.all(got[s, :, n:] == (w[s, :, n:] if in_place else 9.0))
        first = int(b.row_begin[s])
        assert np.array_equal(at[s, :, c:n], np.broadcast_to((np.arange(c, n) if pos is None else pos[first:first + n - c]), at[s, :, c:n].shape)) and np.all(at[s, :, :c] == -7)
        assert np.all(at[s, :, n:] == -7)
    return got


SHAPES = [  # ctx, nodes, page, q_heads, kv_heads, dim
    ([0], [1], 16, 1, 1, 128), ([1], [1], 8, 2, 1, 64), ([127], [1], 16, 8, 1, 128), ([128], [1], 16, 5, 1, 128), ([129], [2], 64, 8, 2, 64),
    ([300], [5], 16, 4, 2, 128), ([255], [16], 32, 8, 1, 128), ([700], [33], 128, 7, 1, 64), ([511], [64], 256, 8, 1, 128), ([900], [70], 16, 12, 2, 128),
    ([5, 0, 130, 64, 900, 1], [3, 1, 0, 16, 7, 40], 16, 6, 2, 128), ([100, 4, 31], [1, 1, 1], 32, 4, 4, 64), ([0], [300], 16, 2, 1, 64),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"case{i}" for i in range(len(SHAPES))])
@pytest.mark.parametrize("kind", ["tree", "causal"])
def test_shapes(gpu, dtype, shape, kind):
    ctx, nodes, page, H, G, D = shape
    b = Batch(700, ctx=ctx, nodes=nodes, page=page, q_heads=H, kv_heads=G, dim=D, dtype=dtype, pad=2)
    check(gpu, b, b.trees(words=5)[0] if kind == "tree" else None, decay=0.75)


@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 64])
def test_heads_sharing_a_kv_head(gpu, group):
    check(gpu, Batch(701, ctx=[200, 33], nodes=[6, 1], page=16, q_heads=2 * group, kv_heads=2, dim=64))


@pytest.mark.parametrize("decay,first_time,in_place", [(1.0, False, True), (0.5, False, False), (0.0, False, True), (1.0, True, False)])
def test_what_positions_had(gpu, decay, first_time, in_place):
    check(gpu, Batch(702, ctx=[70, 3, 0], nodes=[2, 1, 4], page=16, q_heads=4, kv_heads=2, dim=128), decay=decay, first_time=first_time, in_place=in_place)


def test_positions_of_the_rows_layers_and_scale(gpu):
    b = Batch(703, ctx=[20, 3], nodes=[2, 3], page=8, layers=3, q_heads=4, kv_heads=2, dim=64)
    check(gpu, b, layer=2, scale=0.4, pos=np.array([1000, 1001, 2 ** 31 - 1, -5, 0], np.int32))


def test_the_weights_of_all_rows_add_up_to_their_number(gpu):
    b = Batch(704, ctx=[700, 10], nodes=[9, 1], page=16, q_heads=8, kv_heads=2, dim=128, dtype="bfloat16")
    got = check(gpu, b, first_time=True)
    for s in range(2):
        n = int(b.ctx[s] + b.nodes[s])
        assert np.abs(got[s, :, :n].astype(np.float64).sum(-1) - int(b.nodes[s]) * 4).max() <= 4 * int(b.nodes[s]) * 2.0 ** -17


def test_behind_a_prefix_they_add_up_to_less(gpu):
    """lse of an attention over more than these positions."""
    b = Batch(705, ctx=[40], nodes=[3], page=16, q_heads=4, kv_heads=2, dim=64)
    q, _ = inputs(b)
    check(gpu, b, q=q, lse=lse_of(b, 0, q, None, b.dim ** -0.5) + np.float32(2.0))


def test_rows_that_see_nothing_add_nothing(gpu):
    b = Batch(706, ctx=[0, 5], nodes=[3, 2], page=16, q_heads=4, kv_heads=2, dim=64)
    mask = np.zeros((5, 1), np.int64)
    mask[0] = 1
    got = check(gpu, b, mask, first_time=True)
    assert np.all(got[0, :, 1:3] == 0)


@pytest.mark.parametrize("junk", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("nodes", [[1, 3], [40, 2]])
def test_keys_that_a_row_does_not_see_may_be_anything(gpu, junk, nodes):
    b = Batch(707, ctx=[30, 17], nodes=nodes, page=8, q_heads=4, kv_heads=1, dim=64)
    mask, _ = b.trees()
    last = int(b.nodes[0]) - 1
    for i in range(int(b.nodes[0])):
        mask[i, 0] &= ~(1 << last)
    for p in set(range(b.n_pages)) - set(b.table[b.table >= 0].tolist()):
        b.k[:, p] = junk
    for s in range(2):
        n = int(b.ctx[s] + b.nodes[s])
        for j in range(n, -(-n // 8) * 8):
            p, r = b.place(s, j)
            b.k[:, p, :, r] = junk
    clean = Batch.__new__(Batch)
    clean.__dict__.update(b.__dict__)
    clean.k = b.k.copy()
    p, r = b.place(0, 30 + last)
    b.k[:, p, :, r] = junk      # a row that nobody sees
    q, w = inputs(b)
    torch, binding = gpu
    lse = lse_of(clean, 0, q, mask, 0.125)
    k, v, pool = cache_on_gpu(gpu, b)
    out = torch.zeros(w.shape, device="cuda")
    pool.attention_weights(0, batch_on_gpu(gpu, b, None, mask), on_gpu(torch, q).half(), on_gpu(torch, lse), out)
    pool.sync()
    want, bound = _prefix.weights(clean, 0, q, lse, mask, 0.125, None, 1.0)
    n = want.shape[2]
    for s in range(2):
        m = int(b.ctx[s] + b.nodes[s])
        assert np.all(np.abs(out.cpu().numpy()[s, :, :m] - want[s, :, :m]) <= bound[s, :, :m] + 2.0 ** -126)
    assert np.all(out.cpu().numpy()[0, :, 30 + last] == 0) and n


def test_large_scores(gpu):
    """Probabilities from below 2^-126 to 1."""
    b = Batch(708, ctx=[400], nodes=[2], page=16, q_heads=2, kv_heads=1, dim=128)
    q, _ = inputs(b, gain=12.0)
    check(gpu, b, q=q)


def test_many_sequences(gpu):
    rs = np.random.RandomState(9)
    check(gpu, Batch(709, ctx=rs.randint(0, 40, 700), nodes=rs.randint(0, 3, 700), page=8, q_heads=2, kv_heads=1, dim=64, pad=1), decay=0.5)


@pytest.mark.parametrize("nodes", [1, 64, 130])
def test_long_caches(gpu, nodes):
    check(gpu, Batch(710, ctx=[9000], nodes=[nodes], page=64, q_heads=4, kv_heads=1, dim=128, dtype="bfloat16"))


def test_bad_pages_receive_nothing_and_short_arrays_are_reported(gpu):
    torch, binding = gpu
    b = Batch(711, ctx=[40, 300], nodes=[1, 1], page=8, q_heads=2, kv_heads=1, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    q, w = inputs(b)
    lse = lse_of(b, 0, q, None, 0.125)
    want, _ = _prefix.weights(b, 0, q, lse, None, 0.125, w, 0.5)
    table = b.table.copy()
    table[0, 2], table[1, 7] = -1, b.n_pages
    out = torch.full(w.shape, 9.0, device="cuda")
    pool.attention_weights(0, binding.PagedBatch(on_gpu(torch, table), on_gpu(torch, b.row_begin), on_gpu(torch, b.ctx), 2), on_gpu(torch, q).half(), on_gpu(torch, lse), out,
                           weight_in=on_gpu(torch, w), decay=0.5)
    with pytest.raises(binding.PrimaError) as e:
        pool.sync()
    assert "page" in str(e.value)
    got = out.cpu().numpy()
    for s, n, bad in ((0, 41, range(16, 24)), (1, 301, range(56, 64))):
        for j in range(n):
            assert abs(got[s, 0, j] - (w[s, 0, j] * 0.5 if j in bad else want[s, 0, j])) <= 1e-5 * (1 + want[s, 0, j])
    short = torch.full((2, 1, 100), 9.0, device="cuda")
    pool.attention_weights(0, batch_on_gpu(gpu, b), on_gpu(torch, q).half(), on_gpu(torch, lse), short)
    with pytest.raises(binding.PrimaError) as e:
        pool.sync()
    assert "slot" in str(e.value)
    assert np.all(short.cpu().numpy()[0, 0, 41:] == 9.0) and np.all(short.cpu().numpy()[1, 0] != 9.0)


def test_runs_give_the_same_bits_and_a_graph_takes_new_lengths(gpu):
    torch, binding = gpu
    b = Batch(712, ctx=[500, 3, 90], nodes=[3, 1, 20], page=16, q_heads=8, kv_heads=2, dim=128)
    k, v, pool = cache_on_gpu(gpu, b)
    q, w = inputs(b)
    dq, dl, dw = on_gpu(torch, q).half(), on_gpu(torch, lse_of(b, 0, q, None, 128 ** -0.5)), on_gpu(torch, w)
    ctx = on_gpu(torch, b.ctx)
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin), ctx, b.n_tok)
    out, born = torch.zeros_like(dw), torch.zeros(w.shape, dtype=torch.int32, device="cuda")
    pool.attention_weights(0, batch, dq, dl, out, weight_in=dw, born=born)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pool.attention_weights(0, batch, dq, dl, out, weight_in=dw, born=born)
    for lengths in ([500, 3, 90], [0, 0, 0], [17, 2, 91]):
        ctx.copy_(torch.tensor(lengths, dtype=torch.int32))
        want, at = torch.zeros_like(dw), torch.zeros_like(born)
        pool.attention_weights(0, batch, dq, dl, want, weight_in=dw, born=at)
        out.zero_()
        born.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(born, at)
    pool.sync()


def test_argument_errors(gpu):
    torch, binding = gpu
    b = Batch(713, ctx=[4], nodes=[2], page=16, q_heads=4, kv_heads=2, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    batch = batch_on_gpu(gpu, b)
    q, lse, w = torch.zeros((2, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros((2, 4), device="cuda"), torch.zeros((1, 2, 8), device="cuda")
    pool.attention_weights(0, batch, q, lse, w)
    for kw in (dict(layer=1), dict(layer=-1), dict(scale=0.0), dict(scale=float("nan")), dict(decay=-0.1), dict(decay=1.5), dict(decay=float("nan"))):
        args = {"layer": 0, **kw}
        layer = args.pop("layer")
        with pytest.raises(binding.PrimaError) as e:
            pool.attention_weights(layer, batch, q, lse, w, **args)
        assert e.value.code == binding.ERR_ARG
    both = torch.zeros(17, device="cuda")      # overlaps without being the same
    with pytest.raises(binding.PrimaError):
        pool.attention_weights(0, batch, q, lse, both[1:].view(1, 2, 8), weight_in=both[:16].view(1, 2, 8))
    for kw in (dict(lse=lse[:1]), dict(weight=w[:, :1]), dict(weight=w[0]), dict(weight_in=w[..., :4]), dict(born=torch.zeros((1, 2, 8), device="cuda")), dict(q=q.float())):
        args = {"q": q, "lse": lse, "weight": w, **kw}
        with pytest.raises(ValueError):
            pool.attention_weights(0, batch, args.pop("q"), args.pop("lse"), args.pop("weight"), **args)
    pool.sync()
