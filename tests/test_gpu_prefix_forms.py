"""Attention behind shared prefixes: forms in which own positions go through tree attention, and more sequences than are added up one by one."""
import numpy as np
import pytest

from tests import _paged
from tests._prefix import PrefixBatch
from tests.test_gpu_paged import cache_on_gpu, gpu, on_gpu  # noqa: F401
from tests.test_gpu_prefix_attention import check, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("trees", [False, True])
def test_many_rows_with_32_bit_outputs(gpu, dtype, dim, trees):
    b = PrefixBatch(650, [40, 0, 300], [50, 30, 70], [333], [0, 2], 16, layers=2, q_heads=4, kv_heads=2, dim=dim, dtype=dtype, pad=3)
    mask = b.trees(words=2)[0] if trees else None
    check(gpu, b, mask, layer=1, scale=0.2, out_dtype="float32")
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 4, dim)).astype(np.float32), dtype)
    assert np.array_equal(run(gpu, b, mask, q=q)[1], run(gpu, b, mask, q=q, lse=False)[1])


@pytest.mark.parametrize("n", [32768, 32769, 40001])
def test_more_sequences_than_windows(gpu, n):
    """Places are added up for 1024 windows of 32 sequences, of 64 and more beyond 32,768; against tree attention, to which a
    prefix of one page is the first page of every table."""
    torch, binding = gpu
    rs = np.random.RandomState(n)
    nodes = rs.randint(0, 2, n)
    nodes[[0, n - 1]] = 1
    b = PrefixBatch(651, rs.randint(0, 5, n), nodes, [8], [n // 3, n], 8, q_heads=2, kv_heads=1, dim=64)
    k, v, pool = kv = cache_on_gpu(gpu, b)
    q, out, lse = run(gpu, b, pool_kv=kv)
    shared = np.arange(n) >= n // 3
    table = np.where(shared[:, None], np.concatenate([np.repeat(b.prefix_table[:, :1], n, 0), b.table], 1), np.concatenate([b.table, b.table[:, :1]], 1)).astype(np.int32)
    batch = binding.PagedBatch(on_gpu(torch, table), on_gpu(torch, b.row_begin), on_gpu(torch, (b.ctx + 8 * shared).astype(np.int32)), b.n_tok)
    want, z = torch.empty(q.shape, dtype=torch.float16, device="cuda"), torch.empty(q.shape[:2], device="cuda")
    pool.tree_attention(0, batch, on_gpu(torch, q).half(), want, lse=z)
    pool.sync()
    # probabilities and results of both are rounded by half a step each: 2^-11 of values of at most |v|
    assert np.abs(out - want.float().cpu().numpy()).max() <= 4 * 2.0 ** -11 * np.abs(b.v).max()
    assert np.abs(lse - z.cpu().numpy()).max() <= 2.0 ** -18
