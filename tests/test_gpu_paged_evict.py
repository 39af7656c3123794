"""Eviction from the paged cache: choices, moves and refusals, exact."""
import numpy as np
import pytest

from tests import _prefix
from tests._paged import Batch
from tests.test_gpu_paged import cache_on_gpu, gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def arrays(b, spare=3, seed=0):
    rs = np.random.RandomState(seed)
    shape = (b.layers, len(b.ctx), b.kv_heads, int(b.ctx.max()) + spare)
    w = np.exp(rs.standard_normal(shape) * 2).astype(np.float32)
    born = rs.rand(*shape).argsort(-1).astype(np.int32)
    return w, born


def check(gpu, b, keep, w=None, born=None, first=0, recent_from=None, in_place=False, kv=None, length_in_place=False):
    torch, binding = gpu
    k, v, pool = kv or cache_on_gpu(gpu, b)
    if w is None:
        w, born = arrays(b)
    keep = np.broadcast_to(np.array(keep, np.int32), b.ctx.shape).copy()
    recent = None if recent_from is None else np.broadcast_to(np.array(recent_from, np.int32), b.ctx.shape).copy()
    dw, db, length = on_gpu(torch, w), on_gpu(torch, born), on_gpu(torch, b.ctx)
    wo, bo = (dw, db) if in_place else (torch.full_like(dw, 9.0), torch.full_like(db, -9))
    lo = length if length_in_place else torch.full_like(length, -9)
    pool.evict(on_gpu(torch, b.table), length, dw, db, on_gpu(torch, keep), lo, weight_out=wo, born_out=bo, first=first,
               recent_from=None if recent is None else on_gpu(torch, recent))
    pool.sync()
    want_k, want_v = b.k.copy(), b.v.copy()
    want_w, want_b = (w.copy(), born.copy()) if in_place else (np.full_like(w, 9.0), np.full_like(born, -9))
    for layer in range(b.layers):
        for s in range(len(b.ctx)):
            for g in range(b.kv_heads):
                n = int(b.ctx[s])
                _, source = _prefix.choose(w[layer, s, g], born[layer, s, g], n, int(keep[s]), first, None if recent is None else int(recent[s]))
                m = len(source)
                want_w[layer, s, g, :m], want_b[layer, s, g, :m] = w[layer, s, g, source], born[layer, s, g, source]
                for j in np.flatnonzero(source != np.arange(m)):
                    (pt, rt), (pf, rf) = b.place(s, int(j)), b.place(s, int(source[j]))
                    for new, old in ((want_k, b.k), (want_v, b.v)):
                        new[layer, pt, g, rt] = old[layer, pf, g, rf]
    assert np.array_equal(lo.cpu().numpy(), np.minimum(b.ctx, keep))
    assert np.array_equal(wo.cpu().numpy().view(np.uint32), want_w.view(np.uint32)) and np.array_equal(bo.cpu().numpy(), want_b)
    assert np.array_equal(k.float().cpu().numpy(), want_k) and np.array_equal(v.float().cpu().numpy(), want_v)


@pytest.mark.parametrize("dtype,dim,page", [("float16", 128, 16), ("bfloat16", 64, 8), ("float16", 64, 64), ("bfloat16", 128, 32)])
@pytest.mark.parametrize("in_place", [False, True])
def test_types_and_layouts(gpu, dtype, dim, page, in_place):
    b = Batch(800, ctx=[200, 0, 1, 77, 130, 500], nodes=[0] * 6, page=page, layers=3, kv_heads=2, dim=dim, dtype=dtype)
    check(gpu, b, [50, 3, 1, 76, 131, 250], first=4, recent_from=[180, 0, 0, 70, 120, 480], in_place=in_place, length_in_place=in_place)


@pytest.mark.parametrize("keep", [0, 1, 2, 299, 300, 301])
def test_how_many_stay(gpu, keep):
    check(gpu, Batch(801, ctx=[300], nodes=[0], page=16, kv_heads=2, dim=64), keep)


@pytest.mark.parametrize("n", [511, 512, 513, 2047, 2048, 2049, 10000, 10001, 13000, 16384, 16385, 20000])
def test_lengths_around_the_tiles(gpu, n):
    """Up to 16,384 keys stay in shared memory; the others are made again."""
    check(gpu, Batch(802, ctx=[n], nodes=[0], page=32, kv_heads=1, dim=64), n // 3, recent_from=n - 50)


@pytest.mark.parametrize("n", [5000, 17000])
def test_equal_weights_stay_by_slot(gpu, n):
    """Among them more keys with the border's first digit than are set apart (2048)."""
    b = Batch(803, ctx=[n, 90], nodes=[0, 0], page=16, kv_heads=2, dim=64)
    w, born = arrays(b)
    for values in ([1.0], [0.0, -0.0], [3.0, 2.0, 2.0, 2.0, 1.0]):
        w[:] = np.random.RandomState(3).choice(np.array(values, np.float32), w.shape)
        check(gpu, b, [2000, 40], w, born)


def test_odd_weights(gpu):
    """Negative ones, infinities, numbers below the normal ones; NaN is less than any number."""
    b = Batch(804, ctx=[400, 30], nodes=[0, 0], page=16, kv_heads=2, dim=64)
    w, born = arrays(b)
    rs = np.random.RandomState(4)
    w *= rs.choice(np.array([1, -1], np.float32), w.shape)
    for value in (np.inf, -np.inf, np.nan, 1e-42, -1e-42, 0.0):
        w[rs.rand(*w.shape) < 0.1] = value
    for keep in (20, 200, 330, 390):
        check(gpu, b, keep, w, born)
    w[:] = np.nan
    check(gpu, b, 100, w, born)


def test_more_protected_than_stay(gpu):
    b = Batch(805, ctx=[300], nodes=[0], page=16, kv_heads=2, dim=64)
    check(gpu, b, 20, first=50, recent_from=250)
    check(gpu, b, 20, first=10 ** 6)
    check(gpu, b, 100, first=-5, recent_from=2 ** 31 - 1)


def test_one_goes(gpu):
    """A cache that is full drops one entry a step."""
    b = Batch(806, ctx=[257], nodes=[0], page=8, layers=2, kv_heads=4, dim=128)
    check(gpu, b, 256, recent_from=240, in_place=True)


def test_many_choices(gpu):
    rs = np.random.RandomState(6)
    check(gpu, Batch(807, ctx=rs.randint(0, 60, 200), nodes=np.zeros(200, int), page=8, layers=2, kv_heads=2, dim=64), rs.randint(0, 60, 200))


def test_bad_numbers_and_pages_are_skipped(gpu):
    torch, binding = gpu
    b = Batch(808, ctx=[40, 50, 60, 30, 45], nodes=[0] * 5, page=8, kv_heads=1, dim=64)
    w, born = arrays(b, spare=0)
    table = b.table.copy()
    moved = {}
    for s in range(5):
        moved[s] = _prefix.choose(w[0, s, 0], born[0, s, 0], int(b.ctx[s]), 20, 0, None)[1]
    bad_to = int(np.flatnonzero(moved[4] != np.arange(20))[0])      # a slot in front whose page is none
    table[4, bad_to // 8] = b.n_pages + 5
    length, keep = b.ctx.copy(), np.full(5, 20, np.int32)
    length[0], keep[1], length[2] = -3, -1, 10 ** 6
    k, v, pool = cache_on_gpu(gpu, b)
    dw, db = on_gpu(torch, w), on_gpu(torch, born)
    lo = torch.zeros(5, dtype=torch.int32, device="cuda")
    pool.evict(on_gpu(torch, table), on_gpu(torch, length), dw, db, on_gpu(torch, keep), lo)
    with pytest.raises(binding.PrimaError) as e:
        pool.sync()
    assert all(x in str(e.value) for x in ("page", "slot", "length"))
    assert lo.tolist() == [-3, 50, 10 ** 6, 20, 20]
    want = b.k.copy()
    for s in (3, 4):
        for j in np.flatnonzero(moved[s] != np.arange(20)):
            (pt, rt), (pf, rf) = b.place(s, int(j)), b.place(s, int(moved[s][j]))
            if s == 3 or (j // 8 != bad_to // 8 and moved[s][j] // 8 != bad_to // 8):
                want[0, pt, 0, rt] = b.k[0, pf, 0, rf]
    assert np.array_equal(k.float().cpu().numpy(), want)
    assert np.array_equal(dw[0, :3].cpu().numpy(), w[0, :3]) and np.array_equal(dw[0, 3, 0, :20].cpu().numpy(), w[0, 3, 0, moved[3]])


def test_two_streams_and_a_graph(gpu):
    torch, binding = gpu
    b = Batch(809, ctx=[300, 20], nodes=[0, 0], page=16, layers=2, kv_heads=2, dim=64)
    w, born = arrays(b)
    dw, db, length, table = on_gpu(torch, w), on_gpu(torch, born), on_gpu(torch, b.ctx), on_gpu(torch, b.table)
    keep = torch.tensor([100, 15], dtype=torch.int32, device="cuda")
    caches = [cache_on_gpu(gpu, b) for _ in range(3)]

    def call(c, stream=None, outs=None):
        outs = outs or (torch.zeros_like(dw), torch.zeros_like(db), torch.zeros_like(length))
        c[2].evict(table, length, dw, db, keep, outs[2], weight_out=outs[0], born_out=outs[1], recent_from=keep, stream=stream)
        return outs
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    want = call(caches[0])
    given = [tuple(torch.zeros_like(x) for x in want) for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(2):
        call(caches[1 + i], streams[i], given[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, y) for x, y in zip(given[i], want)) and torch.equal(caches[1 + i][0], caches[0][0]) and torch.equal(caches[1 + i][1], caches[0][1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(caches[1], None, given[0])
    for m in (100, 7, 290):
        keep[0] = m
        again, fresh = cache_on_gpu(gpu, b), cache_on_gpu(gpu, b)
        caches[1][0].copy_(again[0])
        caches[1][1].copy_(again[1])
        want = call(fresh)
        for x in given[0]:
            x.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(given[0], want)) and torch.equal(caches[1][0], fresh[0]) and torch.equal(caches[1][1], fresh[1])
    for c in caches:
        c[2].sync()


def test_argument_errors(gpu):
    torch, binding = gpu
    b = Batch(810, ctx=[30], nodes=[0], page=8, kv_heads=2, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    w, born = (on_gpu(torch, x) for x in arrays(b))
    table, length, keep = on_gpu(torch, b.table), on_gpu(torch, b.ctx), torch.tensor([10], dtype=torch.int32, device="cuda")
    lo = torch.zeros_like(length)
    pool.evict(table, length, w.clone(), born.clone(), keep, lo)
    wide = torch.zeros(w.numel() + 1, device="cuda")
    for kw in (dict(weight_out=torch.zeros_like(w)), dict(born_out=torch.zeros_like(born)), dict(workspace=torch.empty(0, dtype=torch.uint8, device="cuda")),
               dict(weight=wide[:-1].view(w.shape), weight_out=wide[1:].view(w.shape), born_out=torch.zeros_like(born))):
        args = {"weight": w, "born": born, **kw}
        with pytest.raises(binding.PrimaError) as e:
            pool.evict(table, length, args.pop("weight"), args.pop("born"), keep, lo, **args)
        assert e.value.code == binding.ERR_ARG
    for kw in (dict(weight=w[0]), dict(born=born.float()), dict(keep=keep.long()), dict(length=length.repeat(2)), dict(weight=w[:, :, :1])):
        args = {"weight": w, "born": born, "keep": keep, "length": length, **kw}
        with pytest.raises(ValueError):
            pool.evict(table, args["length"], args["weight"], args["born"], args["keep"], lo)
    pool.sync()
