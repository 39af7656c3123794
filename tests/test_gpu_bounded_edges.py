"""Operators of long prompts and bounded caches beyond 32-bit offsets, on other streams, with lengths of zero and mixed batches."""
import numpy as np
import pytest

from tests import _paged, _prefix
from tests._paged import Batch
from tests._prefix import PrefixBatch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401
from tests.test_gpu_paged_weights import check as check_weights
from tests.test_gpu_prefix_attention import check as check_prefix, prefix_on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nodes", [[2, 1], [70, 9]], ids=["few rows", "many rows"])
def test_far_pages_give_the_bits_of_near_ones(gpu, nodes):
    """The same entries in the last pages of a cache of more than 2^32 elements per array."""
    torch, binding = gpu
    b = PrefixBatch(900, [200, 37], nodes, [300], [0, 2], 128, dim=128, kv_heads=2, q_heads=8)
    near = cache_on_gpu(gpu, b)
    big = (1 << 17) + 40                      # pages: x 2 heads x 128 x 128 elements = 2^32 and more
    shape = (1, big, 2, 128, 128)
    far_k, far_v = (torch.empty(shape, dtype=torch.float16, device="cuda") for _ in range(2))
    first = big - b.n_pages
    far_k[:, first:], far_v[:, first:] = near[0], near[1]
    far = far_k, far_v, binding.PagedCache(far_k, far_v)
    x = b.rs.standard_normal((b.n_tok, 8 + 4, 128)).astype(np.float32)
    w = np.exp(b.rs.standard_normal((1, 2, 2, 300))).astype(np.float32)
    seen = []
    for (k, v, pool), shift in ((near, 0), (far, first)):
        b.table[b.table >= 0] += shift
        b.prefix_table[b.prefix_table >= 0] += shift
        batch, prefix = batch_on_gpu(gpu, b), prefix_on_gpu(gpu, b)
        dx, gain = on_gpu(torch, x), torch.ones(128, device="cuda")
        q = torch.zeros((b.n_tok, 8, 128), dtype=torch.float16, device="cuda")
        pool.append_norm(0, batch, dx[:, :8], dx[:, 8:10], dx[:, 10:], q, q_gain=gain, k_gain=gain)
        out, lse = torch.zeros_like(q), torch.zeros((b.n_tok, 8), device="cuda")
        pool.prefix_attention(0, batch, prefix, q, out, lse=lse)
        weight, born = on_gpu(torch, w), torch.arange(300, dtype=torch.int32, device="cuda").repeat(1, 2, 2, 1)
        pool.attention_weights(0, batch, q, lse, weight[0], weight_in=weight[0], born=born[0])
        length = on_gpu(torch, b.ctx + b.nodes)
        pool.evict(on_gpu(torch, b.table), length, weight, born, torch.tensor([90, 20], dtype=torch.int32, device="cuda"), length)
        pool.sync()
        seen.append([q, out, lse, weight, born, length, k[:, shift:shift + b.n_pages].clone(), v[:, shift:shift + b.n_pages].clone()])
    for a, c in zip(*seen):
        assert torch.equal(a, c)


def test_weights_of_arrays_beyond_32_bits(gpu):
    """Entries whose offsets pass 2^31, of the last sequence of a long line."""
    torch, binding = gpu
    b = Batch(901, ctx=[5, 70], nodes=[1, 2], page=16, q_heads=4, kv_heads=2, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    stride = (1 << 30) - 5
    q = _paged.rounded(b.rs.standard_normal((3, 4, 64)).astype(np.float32), "float16")
    lse = _paged.attention(b, 0, q, None, 0.125)[1].astype(np.float32)
    near, far = torch.zeros((2, 2, 100), device="cuda"), torch.zeros((2, 2, stride), device="cuda")
    for out in (near, far):
        pool.attention_weights(0, batch_on_gpu(gpu, b), on_gpu(torch, q).half(), on_gpu(torch, lse), out)
    pool.sync()
    assert torch.equal(near, far[..., :100]) and not far[..., 100:].any()


def test_calls_on_a_stream_that_is_not_current(gpu):
    """Tensors of one stream, calls on another that waits for it."""
    torch, binding = gpu
    b = PrefixBatch(902, [60, 5], [2, 1], [500], [0, 2], 16, q_heads=4, kv_heads=2, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    batch, prefix = batch_on_gpu(gpu, b), prefix_on_gpu(gpu, b)
    q = torch.randn((b.n_tok, 4, 64), device="cuda").half()
    w = torch.rand((1, 2, 2, 70), device="cuda")
    seen = []
    side = torch.cuda.Stream()
    for stream in (None, side):
        kk, vv = k.clone(), v.clone()
        mine = binding.PagedCache(kk, vv)
        out, lse, weight, born = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda"), w.clone(), torch.zeros(w.shape, dtype=torch.int32, device="cuda")
        length, keep = on_gpu(torch, b.ctx + b.nodes), torch.tensor([20, 3], dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)
        mine.prefix_attention(0, batch, prefix, q, out, lse=lse, stream=stream)
        mine.attention_weights(0, batch, q, lse, weight[0], weight_in=weight[0], born=born[0], stream=stream)
        mine.evict(on_gpu(torch, b.table), length, weight, born, keep, length, stream=stream)
        mine.sync(stream)
        seen.append([out, lse, weight, born, length, kk, vv])
    for a, c in zip(*seen):
        assert torch.equal(a, c)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [8, 1024, 32768])
@pytest.mark.parametrize("nodes", [1, 45], ids=["few rows", "many rows"])
def test_the_smallest_and_largest_pages(gpu, dim, page, nodes):
    b = PrefixBatch(903, [0, 301, 127], [nodes, 2, nodes], [270], [0, 3], page, q_heads=2, kv_heads=1, dim=dim, dtype="bfloat16")
    check_prefix(gpu, b)
    check_weights(gpu, Batch(904, ctx=[0, 301, 127], nodes=[nodes, 2, nodes], page=page, q_heads=2, kv_heads=1, dim=dim, dtype="bfloat16", spare=1))


@pytest.mark.parametrize("trees", [False, True])
def test_batches_of_long_and_short_requests(gpu, trees):
    """Single tokens, a tree and long chains in one batch; some requests behind a prefix, some alone, some without rows."""
    b = PrefixBatch(905, [900, 3, 0, 40, 260, 1, 15], [1, 40, 0, 3, 1, 17, 0], [700, 30], [0, 3, 5], 16, q_heads=8, kv_heads=1, dim=128, pad=3)
    check_prefix(gpu, b, b.trees()[0] if trees else None)
    b = Batch(906, ctx=[2000, 3, 0, 40, 260, 1, 15], nodes=[1, 60, 0, 3, 1, 17, 0], page=16, q_heads=8, kv_heads=1, dim=128, pad=3)
    check_weights(gpu, b, b.trees()[0] if trees else None)
    b = Batch(907, ctx=[700] + [5] * 60, nodes=[80] + [1] * 60, page=16, q_heads=8, kv_heads=1, dim=64)      # few rows on average
    check_weights(gpu, b, b.trees(words=2)[0] if trees else None)


def test_a_batch_without_rows(gpu):
    """Every row is padding: nothing is written."""
    torch, binding = gpu
    b = PrefixBatch(908, [9, 4], [0, 0], [100], [0, 2], 16, q_heads=2, kv_heads=1, dim=64, pad=3)
    k, v, pool = cache_on_gpu(gpu, b)
    batch = batch_on_gpu(gpu, b)
    q = torch.zeros((3, 2, 64), dtype=torch.float16, device="cuda")
    out, lse, w, born = torch.full_like(q, 7.0), torch.full((3, 2), 7.0, device="cuda"), torch.full((2, 1, 20), 7.0, device="cuda"), torch.full((2, 1, 20), 7, dtype=torch.int32, device="cuda")
    pool.prefix_attention(0, batch, prefix_on_gpu(gpu, b), q, out, lse=lse)
    pool.attention_weights(0, batch, q, lse, w, born=born)
    x = torch.ones((3, 4, 64), device="cuda")
    q_out = torch.full_like(q, 7.0)
    pool.append_norm(0, batch, x[:, :2], x[:, 2:3], x[:, 3:], q_out)
    pool.sync()
    assert (out == 7).all() and (lse == 7).all() and (w == 7).all() and (born == 7).all() and (q_out == 7).all()
    assert np.array_equal(k.float().cpu().numpy(), b.k)


def test_thousands_of_sequences(gpu):
    rs = np.random.RandomState(11)
    n = 2500
    b = PrefixBatch(909, rs.randint(0, 20, n), rs.randint(0, 2, n), [40, 9], [100, 1500, n - 3], 8, q_heads=1, kv_heads=1, dim=64, pad=1)
    check_prefix(gpu, b)
    check_weights(gpu, Batch(910, ctx=rs.randint(0, 20, n), nodes=rs.randint(0, 2, n), page=8, q_heads=1, kv_heads=1, dim=64, pad=1))


def test_bad_rows_are_reported_and_left(gpu):
    torch, binding = gpu
    b = PrefixBatch(911, [20, 9, 5], [2, 2, 2], [50], [0, 3], 16, q_heads=2, kv_heads=1, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    q = torch.randn((6, 2, 64), device="cuda").half()
    prefix = prefix_on_gpu(gpu, b)
    want = torch.zeros_like(q)
    pool.prefix_attention(0, batch_on_gpu(gpu, b), prefix, q, want)
    alone = torch.zeros_like(q)
    pool.tree_attention(0, batch_on_gpu(gpu, b), q, alone)
    pool.sync()
    # Row 1 of the first case lies in the ranges [0, 2) and [1, 6) and has no one value: row_begin has to ascend.
    for begin, ctx, good in (([0, 2, 1, 6], [20, 9, 5], (0,)), ([0, 2, 4, 6], [20, -1, 5], (0, 1, 4, 5)), ([-1, 2, 4, 6], [20, 9, 5], ())):
        batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, np.array(begin, np.int32)), on_gpu(torch, np.array(ctx, np.int32)), 6)
        out, lse, w = torch.full_like(q, 7.0), torch.zeros((6, 2), device="cuda"), torch.full((3, 1, 30), 7.0, device="cuda")
        pool.prefix_attention(0, batch, prefix, q, out, lse=lse)
        with pytest.raises(binding.PrimaError):
            pool.sync()
        for t in good:
            assert (out[t].float() - want[t].float()).abs().max().item() <= 4 * 2.0 ** -11 * np.abs(b.v).max()
        if begin[0] < 0:      # the prefix's own range of rows is bad: it counts as none
            assert (out[:2] == 7).all()
            assert (out[2:].float() - alone[2:].float()).abs().max().item() <= 4 * 2.0 ** -11 * np.abs(b.v).max()
        pool.attention_weights(0, batch, q, lse, w)
        with pytest.raises(binding.PrimaError):
            pool.sync()
        x = torch.ones((6, 4, 64), device="cuda")
        pool.append_norm(0, batch, x[:, :2], x[:, 2:3], x[:, 3:], torch.empty_like(q))
        with pytest.raises(binding.PrimaError):
            pool.sync()
        k.copy_(on_gpu(torch, b.k))
        v.copy_(on_gpu(torch, b.v))


def test_more_rows_than_32_bits_count_are_refused(gpu):
    """Refused by the numbers alone: no array of that size is made, and none is read."""
    import ctypes as C
    torch, binding = gpu
    b = PrefixBatch(912, [4], [2], [20], [0, 1], 16, q_heads=64, kv_heads=1, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    batch, prefix = batch_on_gpu(gpu, b), prefix_on_gpu(gpu, b)
    lib = binding.lib()
    n_tok = 1 << 25
    assert lib.prima_prefix_attention_workspace(pool._h, 1, n_tok, 64) == binding.ERR_ARG
    assert lib.prima_prefix_attention_workspace(pool._h, 1, n_tok - 1, 64) > 0
    desc = binding.PagedBatchDesc.from_buffer_copy(batch.desc)
    desc.n_tok = n_tok
    q = torch.zeros((2, 64, 64), dtype=torch.float16, device="cuda")
    scratch = torch.empty(256, dtype=torch.uint8, device="cuda")
    rc = lib.prima_prefix_attention(pool._h, 0, C.byref(desc), C.byref(prefix.desc), q.data_ptr(), 64, 0.125, q.data_ptr(), 1, None, scratch.data_ptr(), 1 << 62, None)
    assert rc == binding.ERR_ARG and b"2^31" in lib.prima_last_error(None)
    pool.sync()


@pytest.mark.parametrize("n_seq", [2, 63, 64, 65, 600])
def test_evictions_of_many_sequences_in_any_order_of_lengths(gpu, n_seq):
    """Sequences are taken by length up to 64, beyond it as they come; equal lengths, zeros and bad ones among them."""
    from tests.test_gpu_paged_evict import check
    rs = np.random.RandomState(n_seq)
    ctx = rs.randint(0, 60, n_seq)
    ctx[: n_seq // 2] = 37
    check(gpu, Batch(913, ctx=ctx, nodes=[0] * n_seq, page=8, kv_heads=2, dim=64, layers=2), 20)
