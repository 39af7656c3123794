"""Eviction over bad pages: an entry moves whole or not at all."""
import numpy as np
import pytest

from tests import _prefix
from tests._paged import Batch
from tests.test_gpu_paged import cache_on_gpu, gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("bad_source", [False, True])
def test_an_entry_that_cannot_move_keeps_weight_and_position_too(gpu, bad_source, in_place):
    """Keys, values, weights and positions move together or not at all."""
    torch, binding = gpu
    b = Batch(820, ctx=[60, 45], nodes=[0, 0], page=8, kv_heads=2, dim=64, layers=2)
    rs = np.random.RandomState(3)
    w = np.exp(rs.standard_normal((2, 2, 2, 60)) * 2).astype(np.float32)
    born = rs.rand(*w.shape).argsort(-1).astype(np.int32)
    n, m = 60, 20
    sources = [[_prefix.choose(w[i, 0, g], born[i, 0, g], n, m, 0, None)[1] for g in range(2)] for i in range(2)]
    j = int(np.flatnonzero(sources[0][0] != np.arange(m))[0])
    gone = int(sources[0][0][j] if bad_source else j) // 8
    table = b.table.copy()
    table[0, gone] = -5 if bad_source else b.n_pages
    k, v, pool = cache_on_gpu(gpu, b)
    dw, db = on_gpu(torch, w), on_gpu(torch, born)
    wo, bo = (dw, db) if in_place else (torch.full_like(dw, 9.0), torch.full_like(db, -9))
    lo = torch.zeros(2, dtype=torch.int32, device="cuda")
    pool.evict(on_gpu(torch, table), on_gpu(torch, b.ctx), dw, db, torch.tensor([m, 45], dtype=torch.int32, device="cuda"), lo, weight_out=wo, born_out=bo)
    with pytest.raises(binding.PrimaError) as e:
        pool.sync()
    assert "page" in str(e.value) and lo.tolist() == [m, 45]
    got_w, got_b, got_k, got_v = wo.cpu().numpy(), bo.cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy()
    moved, stayed = 0, 0
    want_k, want_v = b.k.copy(), b.v.copy()
    for i in range(2):
        for g in range(2):
            source = sources[i][g].copy()
            lost = (source != np.arange(m)) & ((source // 8 == gone) | (np.arange(m) // 8 == gone))
            source[lost] = np.flatnonzero(lost)
            assert np.array_equal(got_w[i, 0, g, :m], w[i, 0, g, source]) and np.array_equal(got_b[i, 0, g, :m], born[i, 0, g, source])
            for to in np.flatnonzero(source != np.arange(m)):
                (pt, rt), (pf, rf) = b.place(0, int(to)), b.place(0, int(source[to]))
                want_k[i, pt, g, rt], want_v[i, pt, g, rt] = b.k[i, pf, g, rf], b.v[i, pf, g, rf]
                moved += 1
            stayed += int(lost.sum())
    assert moved and stayed and np.array_equal(got_k, want_k) and np.array_equal(got_v, want_v)
