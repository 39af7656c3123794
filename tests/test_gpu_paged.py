"""The paged cache on the GPU: rotation and append, accepted paths, reordering of beams, against 64-bit definitions."""
import numpy as np
import pytest

from tests import _paged
from tests._paged import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2504_08791_b200 import binding
    assert torch.cuda.is_available()
    binding.lib()
    return torch, binding


def on_gpu(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def cache_on_gpu(gpu, b, theta=1e4, mode=0):
    torch, binding = gpu
    dt = getattr(torch, b.dtype)
    k, v = on_gpu(torch, b.k).to(dt), on_gpu(torch, b.v).to(dt)
    return k, v, binding.PagedCache(k, v, rope_theta=theta, rope_mode=mode)


def batch_on_gpu(gpu, b, pos=None, mask=None):
    torch, binding = gpu
    return binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin), on_gpu(torch, b.ctx), b.n_tok,
                              pos=None if pos is None else on_gpu(torch, pos), mask=None if mask is None else on_gpu(torch, mask))


def check_append(gpu, b, src, mode, pos, theta=5e5, layer=0, with_q=True, offset=0, fused=True):
    torch, binding = gpu
    k, v, pool = cache_on_gpu(gpu, b, theta, mode)
    H, G, D = b.q_heads, b.kv_heads, b.dim
    x = _paged.rounded(b.rs.standard_normal((b.n_tok, H + 2 * G, D)).astype(np.float32) * 3, src)
    flat = torch.empty(offset + x.size, dtype=getattr(torch, src), device="cuda")
    dx = flat[offset:].view(b.n_tok, H + 2 * G, D)
    dx.copy_(on_gpu(torch, x))
    parts = dx[:, :H], dx[:, H:H + G], dx[:, H + G:]
    if not fused:
        parts = [p.contiguous() for p in parts]
    q_out = torch.full((b.n_tok, H, D), 7.0, dtype=k.dtype, device="cuda") if with_q else None
    pool.append(layer, batch_on_gpu(gpu, b, pos), parts[0] if with_q else None, parts[1], parts[2], q_out)
    pool.sync()
    where = np.concatenate([b.ctx[s] + np.arange(n) for s, n in enumerate(b.nodes)] + [np.zeros(b.n_tok - b.live, int)]) if pos is None else pos
    want = _paged.rotate(x[:, :H + G], where, theta, mode)
    # products and sum in 32 bits and sine, cosine to 2^-22 each: 2^-20 of both members' magnitudes; then one rounding
    size = np.abs(x[:, :H + G]).astype(np.float64)
    partner = np.roll(size, D // 2, -1) if mode == 0 else size.reshape(*size.shape[:-1], D // 2, 2)[..., ::-1].reshape(size.shape)
    tol = np.abs(want) * _paged.HALF_STEP[b.dtype] + (size + partner) * 2.0 ** -20 + 2.0 ** -25
    new_k, new_v = k.float().cpu().numpy(), v.float().cpu().numpy()
    want_k, want_v = b.k.copy(), b.v.copy()
    for s, n in enumerate(b.nodes):
        for i in range(n):
            page, row = b.place(s, int(b.ctx[s]) + i)
            t = int(b.row_begin[s]) + i
            assert np.all(np.abs(new_k[layer, page, :, row] - want[t, H:]) <= tol[t, H:])
            want_k[layer, page, :, row] = new_k[layer, page, :, row]
            want_v[layer, page, :, row] = _paged.rounded(x[t, H + G:], b.dtype)
    assert np.array_equal(new_k, want_k) and np.array_equal(new_v, want_v)      # nothing else has changed
    if with_q:
        got = q_out.float().cpu().numpy()
        assert np.all(np.abs(got[:b.live] - want[:b.live, :H]) <= tol[:b.live, :H])
        assert np.all(got[b.live:] == 7.0)


@pytest.mark.parametrize("dtype,src", [("float16", "float32"), ("float16", "float16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("dim,mode,page", [(128, 0, 16), (64, 1, 8), (128, 1, 32)])
def test_append_types_and_layouts(gpu, dtype, src, dim, mode, page):
    b = Batch(1, ctx=[0, 7, 16, 31, 100], nodes=[1, 9, 16, 0, 33], page=page, dim=dim, q_heads=6, kv_heads=3, dtype=dtype, layers=2, pad=3)
    check_append(gpu, b, src, mode, None, layer=1)


@pytest.mark.parametrize("offset", [0, 1, 3, 4, 8])
@pytest.mark.parametrize("src", ["float32", "float16"])
def test_append_of_unaligned_sources(gpu, offset, src):
    check_append(gpu, Batch(2, ctx=[5, 40], nodes=[3, 2], page=16, dim=64, q_heads=5, kv_heads=1), src, 0, None, offset=offset)
    check_append(gpu, Batch(2, ctx=[5, 40], nodes=[3, 2], page=16, dim=64, q_heads=5, kv_heads=1), src, 1, None, offset=offset, fused=False)


def test_append_one_token_without_queries_and_many_tokens(gpu):
    check_append(gpu, Batch(3, ctx=[1023], nodes=[1], page=16, dim=128, q_heads=32, kv_heads=8), "float16", 0, None)
    check_append(gpu, Batch(4, ctx=[0], nodes=[1], page=64, dim=64, q_heads=1, kv_heads=1), "float32", 1, None, with_q=False)
    check_append(gpu, Batch(5, ctx=[3] * 70, nodes=[11] * 70, page=32, dim=64, q_heads=4, kv_heads=2, dtype="bfloat16"), "float32", 0, None)


def test_append_positions_of_a_tree_and_far_ones(gpu):
    b = Batch(6, ctx=[10, 20], nodes=[9, 5], page=16, dim=128, q_heads=4, kv_heads=2, dtype="float16", pad=2)
    _, depth = b.trees()
    seq = np.repeat([0, 1], b.nodes)
    pos = np.zeros(b.n_tok, np.int32)
    pos[:b.live] = b.ctx[seq] + depth[:b.live]
    check_append(gpu, b, "float32", 0, pos)
    pos[:b.live] = b.rs.randint(0, 1 << 24, b.live)      # 2^24 turns of the first pair: the fraction is still exact to 2^-25
    check_append(gpu, b, "float32", 0, pos)
    check_append(gpu, b, "float32", 1, pos, theta=1.0)


def test_append_many_sequences(gpu):
    n = 300
    rs = np.random.RandomState(0)
    check_append(gpu, Batch(7, ctx=rs.randint(0, 40, n), nodes=rs.randint(0, 4, n), page=8, dim=64, q_heads=2, kv_heads=1, pad=1), "float16", 0, None)


def test_append_meets_bad_entries(gpu):
    """Rows whose page is no page, or whose slot lies beyond the table, are skipped and reported; the others are written."""
    torch, binding = gpu
    b = Batch(8, ctx=[0, 8, 16], nodes=[4, 4, 4], page=8, dim=64, q_heads=2, kv_heads=1)
    k, v, pool = cache_on_gpu(gpu, b)
    x = b.rs.standard_normal((b.n_tok, 4, 64)).astype(np.float32)
    dx = on_gpu(torch, x)
    q_out = torch.zeros((b.n_tok, 2, 64), dtype=k.dtype, device="cuda")
    for bad, text in ((-1, "page id"), (b.n_pages, "page id"), (2 ** 31 - 1, "page id"), (-2 ** 31, "page id")):
        table = b.table.copy()
        table[1, 1] = bad
        batch = binding.PagedBatch(on_gpu(torch, table), on_gpu(torch, b.row_begin), on_gpu(torch, b.ctx), b.n_tok)
        k.copy_(on_gpu(torch, b.k))
        pool.append(0, batch, dx[:, :2], dx[:, 2:3], dx[:, 3:], q_out)
        with pytest.raises(binding.PrimaError) as e:
            pool.sync()
        assert e.value.code == binding.ERR_DEVICE and text in str(e.value)
        pool.sync()      # reported once
        changed = (k.float().cpu().numpy() != b.k).any(-1)[0]
        want = np.zeros_like(changed)
        for s in (0, 2):
            for i in range(4):
                page, row = b.place(s, int(b.ctx[s]) + i)
                want[page, :, row] = True
        assert np.array_equal(changed, want)
    k.copy_(on_gpu(torch, b.k))
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin), on_gpu(torch, np.array([1 << 20, -5, 2 ** 31 - 3], np.int32)), b.n_tok)
    pool.append(0, batch, dx[:, :2], dx[:, 2:3], dx[:, 3:], q_out)
    with pytest.raises(binding.PrimaError) as e:
        pool.sync()
    assert "slot beyond" in str(e.value) and "length" in str(e.value)
    assert np.array_equal(k.float().cpu().numpy(), b.k)


@pytest.mark.parametrize("dtype,dim,page,layers", [("float16", 128, 16, 3), ("bfloat16", 64, 8, 2), ("float16", 64, 32, 1)])
def test_accept_moves_the_path(gpu, dtype, dim, page, layers):
    torch, binding = gpu
    b = Batch(11, ctx=[0, 7, 30, 1, 64, 9], nodes=[1, 40, 16, 5, 200, 0], page=page, dim=dim, kv_heads=3, dtype=dtype, layers=layers)
    lens = [1, 33, 4, 0, 150, 0]
    path = np.full((6, 160), -9, np.int32)      # what lies behind a path is not read
    for s, n in enumerate(lens):
        path[s, :n] = np.sort(b.rs.permutation(b.nodes[s])[:n])
    path[2, :4] = [0, 1, 7, 15]
    k, v, pool = cache_on_gpu(gpu, b)
    pool.accept(batch_on_gpu(gpu, b), on_gpu(torch, path), on_gpu(torch, np.array(lens, np.int32)))
    pool.sync()
    for got, old in ((k, b.k), (v, b.v)):
        want = old.copy()
        for s, n in enumerate(lens):
            for j in range(n):
                pf, rf = b.place(s, int(b.ctx[s]) + int(path[s, j]))
                pt, rt = b.place(s, int(b.ctx[s]) + j)
                want[:, pt, :, rt] = old[:, pf, :, rf]
        assert np.array_equal(got.float().cpu().numpy(), want)


def test_accept_meets_bad_paths(gpu):
    torch, binding = gpu
    b = Batch(12, ctx=[3, 3], nodes=[6, 6], page=8, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    for path, lens in (([[0, 6], [0, 1]], [2, 2]), ([[-1, 1], [0, 1]], [2, 0]), ([[0, 1], [0, 1]], [3, -1])):
        pool.accept(batch_on_gpu(gpu, b), on_gpu(torch, np.array(path, np.int32)), on_gpu(torch, np.array(lens, np.int32)))
        with pytest.raises(binding.PrimaError) as e:
            pool.sync()
        assert "path" in str(e.value)
    assert np.array_equal(k.float().cpu().numpy()[:, :], b.k)


@pytest.mark.parametrize("dtype,dim,page,keep,beams", [("float16", 128, 16, 4, 4), ("bfloat16", 64, 8, 5, 3), ("float16", 64, 64, 1, 6), ("float16", 128, 8, 3, 1)])
def test_reorder_shares_pages_and_copies_the_last(gpu, dtype, dim, page, keep, beams):
    torch, binding = gpu
    reqs = 3
    b = Batch(21, ctx=np.random.RandomState(1).randint(0, 50, reqs * beams), nodes=[0] * (reqs * beams), page=page, dim=dim, kv_heads=2, dtype=dtype, layers=2,
              spare=reqs * keep + 1)
    length = b.ctx.copy()
    length[0] = 2 * page      # full pages: nothing to copy
    b.table[0, :2] = b.table[0, :2].clip(0)
    used = set(b.table[b.table >= 0].tolist())
    fresh = np.array([p for p in range(b.n_pages) if p not in used][:reqs * keep], np.int32)
    parent = b.rs.randint(0, beams, (reqs, keep)).astype(np.int32)
    parent[0] = 0
    if keep > 1:
        parent[1, :2] = beams - 1
    k, v, pool = cache_on_gpu(gpu, b)
    table_out = torch.full((reqs * keep, b.table.shape[1]), 99, dtype=torch.int32, device="cuda")
    length_out = torch.full((reqs * keep,), 99, dtype=torch.int32, device="cuda")
    pool.reorder(on_gpu(torch, b.table), on_gpu(torch, length), on_gpu(torch, parent), on_gpu(torch, fresh), table_out, length_out)
    pool.sync()
    want_t, want_k, want_v = np.full(table_out.shape, -1, np.int32), b.k.copy(), b.v.copy()
    for r in range(reqs * keep):
        q, j = divmod(r, keep)
        src = q * beams + parent[q, j]
        n = length[src]
        pages = -(-n // page)
        want_t[r, :pages] = b.table[src, :pages]
        if n % page and parent[q, j] in parent[q, :j]:
            want_t[r, pages - 1] = fresh[r]
            for want, old in ((want_k, b.k), (want_v, b.v)):
                want[:, fresh[r], :, :n % page] = old[:, b.table[src, pages - 1], :, :n % page]
        assert int(length_out[r]) == n
    assert np.array_equal(table_out.cpu().numpy(), want_t)
    assert np.array_equal(k.float().cpu().numpy(), want_k) and np.array_equal(v.float().cpu().numpy(), want_v)


def test_reorder_meets_bad_entries(gpu):
    torch, binding = gpu
    b = Batch(22, ctx=[5, 6], nodes=[0, 0], page=8, dim=64, spare=3)
    k, v, pool = cache_on_gpu(gpu, b)
    out, n = torch.zeros((2, b.table.shape[1]), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    for length, parent, fresh, text in (([5, 6], [[0, 2]], [0, 0], "parent"), ([5, 6], [[1, 1]], [0, b.n_pages], "page"), ([-1, 6], [[0, 0]], [0, 1], "length"),
                                        ([1 << 20, 6], [[0, 0]], [0, 1], "length")):
        pool.reorder(on_gpu(torch, b.table), on_gpu(torch, np.array(length, np.int32)), on_gpu(torch, np.array(parent, np.int32)), on_gpu(torch, np.array(fresh, np.int32)), out, n)
        with pytest.raises(binding.PrimaError) as e:
            pool.sync()
        assert text in str(e.value)


def test_argument_errors(gpu):
    torch, binding = gpu
    b = Batch(30, ctx=[4], nodes=[2], page=8, dim=64, q_heads=4, kv_heads=2)
    k, v, pool = cache_on_gpu(gpu, b)
    batch = batch_on_gpu(gpu, b)
    x = torch.zeros((2, 8, 64), dtype=torch.float32, device="cuda")
    q, kk, vv, qo = x[:, :4], x[:, 4:6], x[:, 6:], torch.zeros((2, 4, 64), dtype=k.dtype, device="cuda")
    for call in (lambda: pool.append(1, batch, q, kk, vv, qo), lambda: pool.append(-1, batch, q, kk, vv, qo),
                 lambda: pool.append(0, batch, q.double(), kk.double(), vv.double(), qo), lambda: pool.append(0, batch, q, kk, vv, None),
                 lambda: pool.append(0, batch, q, kk, vv.half(), qo), lambda: pool.append(0, batch, q.bfloat16(), kk.bfloat16(), vv.bfloat16(), qo),
                 lambda: pool.append(0, batch, q, kk[:, :1], vv, qo), lambda: pool.append(0, batch, q[:1], kk, vv, qo), lambda: pool.append(0, batch, q, kk, vv, qo.float()),
                 lambda: pool.append(0, batch, q.transpose(0, 1), kk, vv, qo), lambda: pool.append(0, batch, q.cpu(), kk, vv, qo),
                 lambda: binding.PagedBatch(torch.zeros((1, 2), dtype=torch.int64, device="cuda"), on_gpu(torch, b.row_begin), on_gpu(torch, b.ctx), 2),
                 lambda: binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin)[:1], on_gpu(torch, b.ctx), 2),
                 lambda: pool.accept(batch, torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")),
                 lambda: binding.PagedCache(k[..., :32].contiguous(), v[..., :32].contiguous()), lambda: binding.PagedCache(k.float(), v.float()),
                 lambda: binding.PagedCache(k, v, rope_theta=0.0), lambda: binding.PagedCache(k, v, rope_mode=2), lambda: binding.PagedCache(k, v[:, :1])):
        with pytest.raises((ValueError, binding.PrimaError)):
            call()
    table = on_gpu(torch, b.table)
    n = on_gpu(torch, b.ctx)
    with pytest.raises(binding.PrimaError) as e:
        pool.reorder(table, n, torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), table, n.clone())
    assert "overlap" in str(e.value)
    assert np.array_equal(k.float().cpu().numpy(), b.k)


def test_append_captured_and_replayed_with_new_lengths(gpu):
    """The lengths, tables and positions of a captured call are read when it is replayed; another stream than torch's."""
    torch, binding = gpu
    b = Batch(31, ctx=[4, 20], nodes=[3, 3], page=8, dim=64, q_heads=2, kv_heads=1)
    k, v, pool = cache_on_gpu(gpu, b)
    ctx = on_gpu(torch, b.ctx)
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, b.row_begin), ctx, b.n_tok)
    x = on_gpu(torch, b.rs.standard_normal((6, 4, 64)).astype(np.float32))
    qo = torch.zeros((6, 2, 64), dtype=k.dtype, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        pool.append(0, batch, x[:, :2], x[:, 2:3], x[:, 3:], qo)
    ctx.copy_(torch.tensor([2, 21], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    pool.sync()
    changed = (v.float().cpu().numpy() != b.v).any(-1)[0, :, 0]
    want = np.zeros_like(changed)
    for s, c in enumerate((2, 21)):
        for i in range(3):
            want[b.place(s, c + i)] = True
    assert np.array_equal(changed, want)
    del graph
