"""Attention behind shared prefixes where a score is no number: a NaN stays one and touches no other row."""
import numpy as np
import pytest

from tests import _paged, _prefix
from tests._prefix import PrefixBatch
from tests.test_gpu_paged import gpu  # noqa: F401
from tests.test_gpu_prefix_attention import run

pytestmark = pytest.mark.gpu

BATCHES = {  # own positions, rows, prefix: few rows of a sequence are streamed, many go through tree attention in front
    "whole parts": ([5, 0, 9], [1, 2, 1], 60), "cut prefix": ([5, 0, 9], [1, 2, 1], 9000), "cut own positions": ([4000, 0, 900], [1, 2, 1], 60),
    "all cut": ([3000, 40, 0], [2, 1, 3], 5000), "no prefix": ([5, 700, 0], [1, 2, 1], 0), "many rows": ([5, 0, 300], [40, 50, 3], 700),
    "many rows and no prefix": ([5, 0, 300], [40, 50, 3], 0), "full tiles": ([2] * 40, [4] * 40, 500),
}


def compare(b, got, lse, want, none):
    """Rows of `none` are NaN with a NaN log-sum-exp, all others what they are without any."""
    value, sums, tol, lse_tol = want
    n, half = b.live, _paged.HALF_STEP[b.dtype]
    bad = np.zeros((b.n_tok, b.q_heads), bool)
    bad[tuple(np.array(none).T)] = True
    assert np.all(np.isnan(got[bad])) and np.all(np.isnan(lse[bad]))
    good = ~bad[:n]
    assert np.all((np.abs(got[:n] - value[:n]) <= tol[:n] * (1 + half) + np.abs(value[:n]) * half + 2.0 ** -25)[good])
    empty = np.isneginf(sums[:n])
    assert np.array_equal(np.isneginf(lse[:n])[good], empty[good])
    assert np.all(np.abs(lse[:n] - np.where(empty, 0.0, sums[:n]))[good & ~empty] <= lse_tol[:n][good & ~empty])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("kind", BATCHES)
def test_a_query_without_a_number(gpu, kind, dim):
    ctx, nodes, prefix = BATCHES[kind]
    b = PrefixBatch(630, ctx, nodes, [prefix], [0, len(ctx)], 32, q_heads=6, kv_heads=2, dim=dim)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 6, dim)).astype(np.float32), b.dtype)
    want = _prefix.prefix_attention(b, 0, q, None, dim ** -0.5)
    none = [(0, 1), (b.n_tok - 1, 5), (1, 3)]
    for t, h in none:
        q[t, h, 17] = np.nan
    _, out, lse = run(gpu, b, q=q)
    compare(b, out, lse, want, none)


@pytest.mark.parametrize("prefix", [0, 60, 9000])
@pytest.mark.parametrize("nodes", [[1, 1], [40, 1]], ids=["few rows", "many rows"])
def test_an_own_key_without_a_number(gpu, nodes, prefix):
    """The row's own position is all that it has of its own."""
    b = PrefixBatch(631, [0, 3], nodes, [prefix], [0, 2], 16, q_heads=4, kv_heads=2, dim=64)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 4, 64)).astype(np.float32), b.dtype)
    want = _prefix.prefix_attention(b, 0, q, None, 0.125)
    page, row = b.place(0, 0)
    b.k[0, page, 1, row, 5] = np.nan      # of the second KV head; all rows of the first sequence see it
    _, out, lse = run(gpu, b, q=q)
    compare(b, out, lse, want, [(t, h) for t in range(nodes[0]) for h in (2, 3)])


def test_a_prefix_key_without_a_number(gpu):
    b = PrefixBatch(632, [0, 3, 2], [1, 2, 1], [1, 300], [0, 1, 2], 16, q_heads=4, kv_heads=2, dim=64)
    q = _paged.rounded(b.rs.standard_normal((b.n_tok, 4, 64)).astype(np.float32), b.dtype)
    want = _prefix.prefix_attention(b, 0, q, None, 0.125)
    b.k[0, b.prefix_table[0, 0], 0, 0, 9] = np.nan      # the first prefix is this position alone
    b.k[0, b.prefix_table[1, 3], 1, 2, 9] = np.nan
    _, out, lse = run(gpu, b, q=q)
    compare(b, out, lse, want, [(0, 0), (0, 1)] + [(t, h) for t in (1, 2) for h in (2, 3)])
