"""The paged cache's calls where they are least at home: caches beyond 32 bits, captured calls, arrays of another kind."""
import ctypes

import numpy as np
import pytest

from paper_2504_08791_b200 import synth
from tests import _paged
from tests._paged import Batch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401
from tests.test_gpu_paged_decoding import load, stepper
from tests.test_gpu_tree_attention import check as check_attention

pytestmark = pytest.mark.gpu


def i32(torch, x):
    return on_gpu(torch, np.array(x, np.int32))


@pytest.mark.parametrize("nodes", [[2, 1], [70, 9]], ids=["few rows", "many rows"])
def test_far_pages_give_the_bits_of_near_ones(gpu, nodes):
    """The same entries in the last pages of a cache of more than 2^32 elements per array."""
    torch, binding = gpu
    b = Batch(300, ctx=[200, 37], nodes=nodes, page=128, dim=128, kv_heads=2, q_heads=8, spare=4)
    free = [p for p in range(b.n_pages) if p not in set(b.table[b.table >= 0].tolist())]
    x = b.rs.standard_normal((b.n_tok, 8 + 4, 128)).astype(np.float32)
    mask = b.trees(words=2)[0]
    path, path_len = np.array([[0, 1], [0, 0]], np.int32), np.array([2 if nodes[0] == 2 else 1, 1], np.int32)
    if nodes[0] > 2:
        path[0] = [3, 50]
        path_len[0] = 2
    near = cache_on_gpu(gpu, b)
    big = (1 << 17) + 40                      # pages: x 2 heads x 128 x 128 elements = 2^32 and more
    assert big * 2 * 128 * 128 > 1 << 32
    shape = (1, big, 2, 128, 128)
    far_k, far_v = (torch.empty(shape, dtype=torch.float16, device="cuda") for _ in range(2))
    first = big - b.n_pages
    far_k[:, first:], far_v[:, first:] = near[0], near[1]
    far = far_k, far_v, binding.PagedCache(far_k, far_v)
    seen = []
    for (k, v, pool), shift in ((near, 0), (far, first)):
        b.table[b.table >= 0] += shift
        batch = batch_on_gpu(gpu, b, mask=mask)
        dx = on_gpu(torch, x)
        q = torch.zeros((b.n_tok, 8, 128), dtype=torch.float16, device="cuda")
        pool.append(0, batch, dx[:, :8], dx[:, 8:10], dx[:, 10:], q)
        out = torch.zeros_like(q)
        pool.tree_attention(0, batch, q, out)
        pool.accept(batch, on_gpu(torch, path), on_gpu(torch, path_len))
        table, length = torch.zeros((3, b.table.shape[1]), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
        pool.reorder(on_gpu(torch, b.table), i32(torch, [202, 38]), i32(torch, [[0, 1, 0]]), i32(torch, np.array(free[:3]) + shift), table, length)
        pool.sync()
        table[table >= 0] -= shift
        seen.append([q, out, k[:, shift:shift + b.n_pages].clone(), v[:, shift:shift + b.n_pages].clone(), table, length])
    for a, c in zip(*seen):
        assert torch.equal(a, c)


def test_accept_and_reorder_captured_and_replayed(gpu):
    """Paths, parents and lengths of a captured call are read when it is replayed."""
    torch, binding = gpu
    b = Batch(301, ctx=[5, 20], nodes=[6, 6], page=8, dim=64, kv_heads=2, layers=2, spare=4)
    free = [p for p in range(b.n_pages) if p not in set(b.table[b.table >= 0].tolist())]
    k, v, pool = cache_on_gpu(gpu, b)
    batch = batch_on_gpu(gpu, b)
    table = on_gpu(torch, b.table)
    path, path_len, parent, length, fresh = i32(torch, [[0, 1], [0, 1]]), i32(torch, [0, 0]), i32(torch, [[0, 1]]), i32(torch, [1, 1]), i32(torch, free[:2])
    table_out, length_out = torch.zeros_like(table), torch.zeros_like(length)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pool.accept(batch, path, path_len)
        pool.reorder(table, length, parent, fresh, table_out, length_out)
    path.copy_(i32(torch, [[0, 2], [1, 4]]))
    path_len.copy_(i32(torch, [2, 2]))
    parent.copy_(i32(torch, [[1, 1]]))
    length.copy_(i32(torch, [7, 22]))
    graph.replay()
    pool.sync()
    want = b.k.copy()
    for s, j, a in ((0, 1, 2), (1, 0, 1), (1, 1, 4)):
        (pf, rf), (pt, rt) = b.place(s, int(b.ctx[s]) + a), b.place(s, int(b.ctx[s]) + j)
        want[:, pt, :, rt] = b.k[:, pf, :, rf]
    last = b.table[1, 2]
    want[:, free[1], :, :6] = want[:, last, :, :6]
    assert np.array_equal(k.float().cpu().numpy(), want)
    want_t = np.full_like(b.table, -1)
    want_t[:, :3] = b.table[1, :3]
    want_t[1, 2] = free[1]
    assert np.array_equal(table_out.cpu().numpy(), want_t) and length_out.tolist() == [22, 22]
    del graph


def test_window_captured_after_its_first_call(gpu):
    """The first call on a context allocates and is refused under capture, with nothing broken; a later one is captured
    and replayed with other rows and lengths, giving the bits of the plain call."""
    torch, binding = gpu
    cfg = synth.model_config("tiny", max_n_tok=4)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = load(gpu, cfg, 47)
        m = stepper(gpu, ctx, page=8)
    L = cfg["n_layers"]
    with torch.cuda.stream(stream):
        pages = []
        m.pages.grow(pages, 16)
        length = i32(torch, [0])
        batch = binding.PagedBatch(m.table_of([pages]), i32(torch, [0, 2]), length, 2)
        hid, out = torch.zeros((2, cfg["hidden"]), device="cuda"), torch.zeros((2, cfg["hidden"]), device="cuda")
        rows = [torch.randn((2, cfg["hidden"]), device="cuda") for _ in range(2)]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out.zero_()
            with pytest.raises(binding.PrimaError) as e:
                ctx.forward_window_paged(m.pool, 0, L, hid, out, batch)
        assert e.value.code == binding.ERR_STATE
        want = []
        for i in range(2):
            length.fill_(2 * i)
            hid.copy_(rows[i])
            ctx.forward_window_paged(m.pool, 0, L, hid, out, batch)
            want.append(out.clone())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.forward_window_paged(m.pool, 0, L, hid, out, batch)
        for i in range(2):
            length.fill_(2 * i)
            hid.copy_(rows[i])
            out.zero_()
            graph.replay()
            assert torch.equal(out, want[i])
        m.pool.sync()
        torch.cuda.synchronize()
        del graph
    ctx.close()


def test_arrays_that_are_not_aligned_or_too_many(gpu):
    torch, binding = gpu
    b = Batch(302, ctx=[4], nodes=[2], page=8, dim=64, q_heads=4, kv_heads=2)
    k, v, pool = cache_on_gpu(gpu, b)
    L, h = binding.lib(), pool._h
    a = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda").data_ptr()
    ws = binding.lib().prima_tree_attention_workspace(h, 1, 2, 4)
    work = torch.zeros(ws, dtype=torch.uint8, device="cuda").data_ptr()
    good = [1, 2, a, a, a, 4, None, None, 0]

    def desc(**change):
        names = [n for n, _ in binding.PagedBatchDesc._fields_]
        return ctypes.byref(binding.PagedBatchDesc(*[change.get(n, x) for n, x in zip(names, good)]))
    append = [h, 0, desc(), a, a, a, 0, 4, 512, 512, 512, a, None]
    attend = [h, 0, desc(), a, 4, 1.0, a, 1, None, work, ws, None]
    accept = [h, desc(), a, a, 2, None]
    reorder = [h, 1, 1, 1, a, 1, a + 64, a, a, a + 4096, a + 8192, None]
    for bad in (dict(row_begin=a + 2), dict(ctx_len=a + 1), dict(table=a + 2), dict(pos=a + 2), dict(mask=a + 4, mask_words=1), dict(table_stride=1 << 31), dict(table_stride=0)):
        for call, args, at in ((L.prima_paged_append, append, 2), (L.prima_tree_attention, attend, 2), (L.prima_paged_accept, accept, 1)):
            args = list(args)
            args[at] = desc(**bad)
            assert call(*args) == binding.ERR_ARG, bad
    for call, args, changes in ((L.prima_paged_append, append, ((3, a + 2), (4, a + 1), (5, a + 2), (11, a + 8))), (L.prima_tree_attention, attend, ((3, a + 2), (6, a + 8), (8, a + 2), (9, work + 16))),
                                (L.prima_paged_accept, accept, ((2, a + 2), (3, a + 1))),
                                (L.prima_paged_reorder, reorder, ((4, a + 2), (6, a + 65), (7, a + 1), (8, a + 2), (9, a + 4098), (10, a + 8193), (5, 1 << 31)))):
        for at, x in changes:
            bad = list(args)
            bad[at] = x
            assert call(*bad) == binding.ERR_ARG, (call.__name__, at)
    pool.sync()
    assert np.array_equal(k.float().cpu().numpy(), b.k)


def test_workspaces_of_the_caller(gpu):
    """Any contiguous tensor of enough bytes on the right device; nothing else."""
    torch, binding = gpu
    b = Batch(303, ctx=[100], nodes=[3], page=16, dim=64, q_heads=4, kv_heads=2)
    k, v, pool = cache_on_gpu(gpu, b)
    batch = batch_on_gpu(gpu, b)
    q = on_gpu(torch, _paged.rounded(b.rs.standard_normal((3, 4, 64)).astype(np.float32), b.dtype)).to(k.dtype)
    want, out = torch.zeros_like(q), torch.zeros_like(q)
    pool.tree_attention(0, batch, q, want)
    n = pool.tree_attention_workspace(batch, 4).numel()
    pool.tree_attention(0, batch, q, out, workspace=torch.empty(-(-n // 8), dtype=torch.int64, device="cuda"))
    assert torch.equal(out, want)
    with pytest.raises(ValueError):
        pool.tree_attention(0, batch, q, out, workspace=torch.empty(n, dtype=torch.uint8))
    with pytest.raises(ValueError):
        pool.tree_attention(0, batch, q, out, workspace=torch.empty((n, 2), dtype=torch.uint8, device="cuda")[:, 0])
    with pytest.raises(binding.PrimaError):
        pool.tree_attention(0, batch, q, out, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
    logits, cum = torch.randn((1, 2, 50), device="cuda"), torch.zeros((1, 2), device="cuda")
    score, parent, token = torch.zeros((1, 4), device="cuda"), *(torch.zeros((1, 4), dtype=torch.int32, device="cuda") for _ in range(2))
    n = binding.prima_beam_select_workspace(1, 2, 50, 4).numel()
    with pytest.raises(ValueError):
        binding.prima_beam_select(logits, cum, score, parent, token, workspace=torch.empty(n, dtype=torch.uint8))
    with pytest.raises(binding.PrimaError):
        binding.prima_beam_select(logits, cum, score, parent, token, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))


def test_first_beams_of_requests(gpu):
    """The slice of one beam per request (as after a prompt) is taken in place."""
    torch, binding = gpu
    logits = torch.randn((3, 4, 1000), device="cuda")
    cum = torch.zeros((3, 1), device="cuda")
    both = []
    for x in (logits[:, :1], logits[:, :1].contiguous()):
        out = torch.zeros((3, 5), device="cuda"), *(torch.zeros((3, 5), dtype=torch.int32, device="cuda") for _ in range(2))
        binding.prima_beam_select(x, cum, *out)
        both.append(out)
    for a, c in zip(*both):
        assert torch.equal(a, c)
    assert torch.equal(both[0][2], torch.topk(logits[:, 0], 5).indices.int())


def test_steps_of_a_context_on_its_own_stream(gpu):
    """A prompt of many steps, queued from torch's default stream while the context's own stream is still busy: the
    small arrays of a step must not be overwritten by a later one's before it has read them."""
    torch, binding = gpu
    from paper_2504_08791_b200.paged import BeamDecoder, PagedStepper
    cfg = synth.model_config("tiny", max_n_tok=4)
    prompt = [int(x) for x in np.random.RandomState(5).randint(0, cfg["vocab"], 37)]
    stream = torch.cuda.Stream()
    seen = []
    for own in (None, stream):
        ctx = binding.Context(cfg, stream=own)
        for layer, tid, rows, cols, data in synth.iter_model_tensors(48, cfg):
            ctx.load(layer, tid, data, rows, cols)
        shape = (cfg["n_layers"], 64, cfg["n_kv_heads"], 8, cfg["head_dim"])
        k, v = (torch.zeros(shape, dtype=torch.float16, device="cuda") for _ in range(2))
        torch.cuda.synchronize()
        m = PagedStepper(ctx, k, v)
        with torch.cuda.stream(own):
            torch.cuda._sleep(50_000_000)      # some 25 ms
        pages = []
        m.prefill(prompt, pages)
        torch.cuda.synchronize()
        m.pool.sync()
        seen.append([m.logits[:1].clone(), k[:, pages].clone(), v[:, pages].clone(), BeamDecoder(m, 3).generate(prompt, 4)])
        assert len(m.pages.free) == 64 - len(pages)
        ctx.close()
    assert all(torch.equal(a, b) for a, b in zip(seen[0][:3], seen[1][:3])) and seen[0][3] == seen[1][3]


def test_a_full_cache_leaves_no_page_behind(gpu):
    torch, binding = gpu
    from paper_2504_08791_b200.paged import BeamDecoder
    cfg = synth.model_config("tiny", max_n_tok=4)
    ctx = load(gpu, cfg, 49)
    m = stepper(gpu, ctx, n_pages=9, page=8)
    prompt = [int(x) for x in np.random.RandomState(6).randint(0, cfg["vocab"], 20)]
    with pytest.raises(RuntimeError) as e:
        BeamDecoder(m, 4).generate(prompt, 40)
    assert "full" in str(e.value) and len(m.pages.free) == 9
    ctx.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [8, 1024, 32768])
@pytest.mark.parametrize("nodes", [3, 45, 260], ids=["few rows", "one tile", "several tiles"])
def test_attention_over_the_smallest_and_largest_pages(gpu, dim, page, nodes):
    b = Batch(304, ctx=[0, 301, 127], nodes=[nodes, 2, nodes], page=page, q_heads=2, kv_heads=1, dim=dim, dtype="bfloat16", spare=1)
    check_attention(gpu, b, b.trees(words=5)[0])
    check_attention(gpu, b, None)


@pytest.mark.parametrize("rows", [1, 40])
def test_attention_of_thousands_of_sequences(gpu, rows):
    n = 3000 if rows == 1 else 400
    rs = np.random.RandomState(8)
    b = Batch(305, ctx=rs.randint(0, 40, n), nodes=rs.randint(0, rows + 1, n) if rows == 1 else np.full(n, rows), page=8, q_heads=1, kv_heads=1, dim=64, pad=1)
    check_attention(gpu, b, None)


def test_accept_reports_paths_that_do_not_ascend(gpu):
    torch, binding = gpu
    b = Batch(13, ctx=[3, 3], nodes=[6, 6], page=8, dim=64)
    for path, moved in (([2, 1, 4], {0: 2, 2: 4}), ([1, 1, 3], {0: 1, 2: 3}), ([0, 3, 2], {1: 3})):
        k, v, pool = cache_on_gpu(gpu, b)
        pool.accept(batch_on_gpu(gpu, b), on_gpu(torch, np.array([path, [1, 2, 5]], np.int32)), on_gpu(torch, np.array([3, 3], np.int32)))
        with pytest.raises(binding.PrimaError) as e:
            pool.sync()
        assert "path" in str(e.value)
        for got, old in ((k, b.k), (v, b.v)):
            want = old.copy()
            for s, moves in ((0, moved), (1, {0: 1, 1: 2, 2: 5})):
                for j, a in moves.items():
                    (pf, rf), (pt, rt) = b.place(s, 3 + a), b.place(s, 3 + j)
                    want[:, pt, :, rt] = old[:, pf, :, rf]
            assert np.array_equal(got.float().cpu().numpy(), want)


def test_reorder_gives_rows_of_bad_parents_no_pages(gpu):
    """Such a row would share the partly filled page of another one, and both would append to it."""
    torch, binding = gpu
    b = Batch(23, ctx=[13, 6], nodes=[0, 0], page=8, dim=64, spare=5)
    used = set(b.table[b.table >= 0].tolist())
    fresh = np.array([p for p in range(b.n_pages) if p not in used][:4], np.int32)
    k, v, pool = cache_on_gpu(gpu, b)
    for parent in ([0, -1, 1, 2], [-1, 0, 5, 1]):
        out, n = torch.full((4, b.table.shape[1]), 99, dtype=torch.int32, device="cuda"), torch.full((4,), 99, dtype=torch.int32, device="cuda")
        pool.reorder(on_gpu(torch, b.table), on_gpu(torch, b.ctx), on_gpu(torch, np.array([parent], np.int32)), on_gpu(torch, fresh), out, n)
        with pytest.raises(binding.PrimaError) as e:
            pool.sync()
        assert "parent" in str(e.value)
        for r, p in enumerate(parent):
            good = p in (0, 1)
            assert int(n[r]) == (b.ctx[p] if good else 0)
            want = b.table[p].copy() if good else np.full(b.table.shape[1], -1, np.int32)
            assert np.array_equal(out[r].cpu().numpy(), want)
    assert np.array_equal(k.float().cpu().numpy(), b.k) and np.array_equal(v.float().cpu().numpy(), b.v)


def test_sync_of_one_stream_keeps_what_another_raises(gpu):
    """One thread meets bad slots on its stream and reports them without end; what another thread meets on another stream is
    reported by one of the calls that begin after it."""
    import threading
    import time
    torch, binding = gpu
    b = Batch(32, ctx=[4], nodes=[1], page=8, dim=64, q_heads=2, kv_heads=1)
    k, v, pool = cache_on_gpu(gpu, b)
    x = torch.zeros((1, 1, 64), device="cuda")
    one = on_gpu(torch, b.row_begin)
    slot = binding.PagedBatch(on_gpu(torch, b.table), one, on_gpu(torch, np.array([1000], np.int32)), 1)
    page = binding.PagedBatch(torch.full_like(on_gpu(torch, b.table), -1), one, on_gpu(torch, b.ctx), 1)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    calls, told, stop, failed = [0], [], [], []

    def report():
        try:
            while not stop:
                pool.append(0, slot, None, x, x, stream=streams[0])
                try:
                    pool.sync(streams[0])
                except binding.PrimaError as e:
                    if "page" in str(e):
                        told.append(1)
                calls[0] += 1
        except BaseException as e:
            failed.append(e)
    thread = threading.Thread(target=report)
    thread.start()
    try:
        lost = 0
        for i in range(2000):
            told.clear()
            pool.append(0, page, None, x, x, stream=streams[1])
            streams[1].synchronize()
            want, end = calls[0] + 2, time.monotonic() + 20
            while calls[0] < want and not failed and time.monotonic() < end:
                time.sleep(0)
            assert calls[0] >= want
            lost += not told
    finally:
        stop.append(1)
        thread.join()
    assert not failed and lost == 0


def test_a_context_made_on_a_side_stream_and_used_outside_of_it(gpu):
    """Its steps run on the stream that was current when it was made; selection, reordering and accepted paths follow them,
    though another stream is current."""
    torch, binding = gpu
    from paper_2504_08791_b200.paged import BeamDecoder, DraftTree, TreeSpeculativeDecoder
    cfg = synth.model_config("tiny", max_n_tok=4)
    prompt = [int(x) for x in np.random.RandomState(7).randint(0, cfg["vocab"], 9)]
    side, seen = torch.cuda.Stream(), []

    def propose(history, limit):
        return DraftTree([history[-1], history[-2], 3, 4], [-1, 0, 0, 2])
    for made_on in (None, side):
        with torch.cuda.stream(made_on):
            ctx = load(gpu, cfg, 50)
            m = stepper(gpu, ctx, page=8)
        torch.cuda.synchronize()
        with torch.cuda.stream(made_on):
            torch.cuda._sleep(50_000_000)      # some 25 ms
        beams = BeamDecoder(m, 3).generate(prompt, 5)
        pages = []
        m.prefill(prompt[:-1], pages)
        out, _ = TreeSpeculativeDecoder(m, propose).generate(prompt, pages, len(prompt) - 1, 6)
        torch.cuda.synchronize()
        m.pool.sync()
        seen.append((beams, out))
        ctx.close()
    assert seen[0] == seen[1]
