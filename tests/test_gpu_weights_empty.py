"""Attention weights where a row is marked as one that sees nothing: it adds nothing, whatever its query holds."""
import numpy as np
import pytest

from tests import _paged, _prefix
from tests._paged import Batch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("junk", [np.nan, np.inf])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes,group", [([3, 1], 2), ([3, 1], 4), ([9, 1], 4), ([30, 2], 8), ([100, 2], 8), ([5, 40], 1)])
def test_a_row_whose_sum_is_that_of_nothing_adds_nothing(gpu, nodes, group, dim, junk):
    """Whatever its query holds; the rows beside it are as without it."""
    torch, binding = gpu
    b = Batch(821, ctx=[150, 33], nodes=nodes, page=16, q_heads=2 * group, kv_heads=2, dim=dim)
    k, v, pool = cache_on_gpu(gpu, b)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, b.q_heads, dim)).astype(np.float32), b.dtype)
    lse = _paged.attention(b, 0, q, None, dim ** -0.5)[1].astype(np.float32)
    for t, h in ((0, 0), (1, 2 * group - 1), (nodes[0] - 1, group), (b.n_tok - 1, 0)):
        lse[t, h] = -np.inf
    want, bound = _prefix.weights(b, 0, q, lse, None, dim ** -0.5, None, 1.0)      # leaves these rows out
    q[np.isneginf(lse)] = junk
    out = torch.zeros(want.shape, device="cuda")
    pool.attention_weights(0, batch_on_gpu(gpu, b), on_gpu(torch, q).half(), on_gpu(torch, lse), out)
    pool.sync()
    got = out.cpu().numpy()
    for s in range(2):
        n = int(b.ctx[s] + b.nodes[s])
        assert np.all(np.abs(got[s, :, :n] - want[s, :, :n]) <= bound[s, :, :n] + 2.0 ** -126)
