"""Sequences with bad numbers are left as they were by every operator of a bounded cache, the good ones beside them are served."""
import numpy as np
import pytest

from tests import _paged, _prefix
from tests._paged import Batch
from tests.test_gpu_paged import cache_on_gpu, gpu, on_gpu  # noqa: F401
from tests.test_gpu_paged_evict import check as check_evict
from tests.test_gpu_paged_weights import lse_of

pytestmark = pytest.mark.gpu


# row_begin, ctx_len, sequences that are good
CASES = {"a negative length": ([0, 2, 4, 6], [20, -1, 5], (0, 2)), "rows behind the end": ([0, 2, 4, 9], [20, 9, 5], (0, 1)), "a negative first row": ([-1, 2, 4, 6], [20, 9, 5], (1, 2))}


@pytest.mark.parametrize("heads", [2, 24], ids=["few rows", "many rows"])
@pytest.mark.parametrize("case", CASES)
def test_weights_of_bad_sequences_are_left(gpu, case, heads):
    torch, binding = gpu
    begin, ctx, good = CASES[case]
    b = Batch(830, [20, 9, 5], [2, 2, 2], 16, q_heads=heads, kv_heads=1, dim=64)
    k, v, pool = cache_on_gpu(gpu, b)
    q = _paged.rounded(b.rs.standard_normal((6, heads, 64)).astype(np.float32), b.dtype)
    lse = lse_of(b, 0, q, None, 0.125)
    want, bound = _prefix.weights(b, 0, q, lse, None, 0.125, None, 1.0)
    w, born = torch.full((3, 1, 30), 7.0, device="cuda"), torch.full((3, 1, 30), -7, dtype=torch.int32, device="cuda")
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, np.array(begin, np.int32)), on_gpu(torch, np.array(ctx, np.int32)), 6)
    pool.attention_weights(0, batch, on_gpu(torch, q).half(), on_gpu(torch, lse), w, born=born)
    with pytest.raises(binding.PrimaError):
        pool.sync()
    got, at = w.cpu().numpy(), born.cpu().numpy()
    for s in range(3):
        n = int(b.ctx[s] + 2) if s in good else 0
        assert np.all(np.abs(got[s, :, :n] - want[s, :, :n]) <= bound[s, :, :n] + 2.0 ** -126) and np.all(got[s, :, n:] == 7.0)
        assert np.all(at[s, 0, n:] == -7) and (not n or at[s, 0, n - 2:n].tolist() == [n - 2, n - 1])


@pytest.mark.parametrize("rows", [2, 300], ids=["few rows", "many rows"])
@pytest.mark.parametrize("case", CASES)
def test_rows_of_bad_sequences_are_not_appended(gpu, case, rows):
    torch, binding = gpu
    begin, ctx, good = CASES[case]
    b = Batch(831, [20, 9, 5], [rows] * 3, 16, q_heads=2, kv_heads=1, dim=64)
    begin = [x // 2 * rows if x > 0 else x for x in begin[:3]] + [begin[3] if begin[3] == 9 and rows == 2 else 3 * rows + (5 if begin[3] == 9 else 0)]
    k, v, pool = cache_on_gpu(gpu, b)
    x, q, gain = torch.randn((3 * rows, 4, 64), device="cuda"), torch.full((3 * rows, 2, 64), 7.0, dtype=torch.float16, device="cuda"), torch.ones(64, device="cuda")
    batch = binding.PagedBatch(on_gpu(torch, b.table), on_gpu(torch, np.array(begin, np.int32)), on_gpu(torch, np.array(ctx, np.int32)), 3 * rows)
    pool.append_norm(0, batch, x[:, :2], x[:, 2:3], x[:, 3:], q, q_gain=gain, k_gain=gain)
    changed, kk, vv = [], k.float().cpu().numpy(), v.float().cpu().numpy()
    # A row asks for its own sequence alone: one whose range ends behind the last row serves the rows that are there.
    served = set(good) | ({2} if case == "rows behind the end" else set())
    if case != "rows behind the end":
        with pytest.raises(binding.PrimaError):
            pool.sync()
    for s in range(3):
        rows_of = q[s * rows:(s + 1) * rows]
        assert (rows_of != 7.0).any() if s in served else (rows_of == 7.0).all()
        for i in range(rows):
            page, row = b.place(s, int(b.ctx[s]) + i)
            same = np.array_equal(kk[0, page, :, row], b.k[0, page, :, row]) and np.array_equal(vv[0, page, :, row], b.v[0, page, :, row])
            assert same != (s in served)
            changed.append((page, row))
    touched = np.ones(b.k.shape[:4], bool)
    for page, row in changed:
        touched[:, page, :, row] = False
    assert np.array_equal(kk[touched], b.k[touched]) and np.array_equal(vv[touched], b.v[touched])


@pytest.mark.parametrize("equal", [2047, 2048, 2049])
def test_as_many_keys_as_are_set_apart(gpu, equal):
    """`equal` keys share the border's first digit (2048 are set apart), with different lower digits; the others lie above and below."""
    n, above = 4000, 700
    b = Batch(832, ctx=[n], nodes=[0], page=32, kv_heads=1, dim=64)
    rs = np.random.RandomState(equal)
    w = np.full(n, 0.25, np.float32)
    w[:above] = 4.0
    # a digit of 11 bits: sign, exponent, two bits of the significand; 1.0 to below 1.25 is one of them
    w[above:above + equal] = 1.0 + rs.randint(0, 1 << 21, equal).astype(np.float32) * np.float32(2.0 ** -23)
    w = rs.permutation(w).reshape(1, 1, 1, n)
    born = rs.permutation(n).astype(np.int32).reshape(1, 1, 1, n)
    for keep in (above + 1, above + equal // 2, above + equal - 1):
        check_evict(gpu, b, keep, w, born)
