"""Attention behind shared prefixes whose tiles follow one another in every order: full ones, small ones, of one unit and more."""
import numpy as np
import pytest

from tests._prefix import PrefixBatch
from tests.test_gpu_paged import gpu  # noqa: F401
from tests.test_gpu_prefix_attention import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("longest", [100, 600])
def test_tiles_of_every_kind_behind_one_another(gpu, dim, longest):
    """Three times as many (prefix, KV head) as CTAs, so that each passes through full tiles, which both accumulators share,
    and small ones, of which the second accumulator has no unit where there is only one."""
    rs = np.random.RandomState(longest)
    n = 220
    nodes = np.where(np.arange(n) % 3 == 0, rs.randint(17, 33, n), 1)      # 8 query heads a KV head: 136 to 256 rows, or 8
    b = PrefixBatch(620, rs.randint(0, 4, n), nodes, rs.randint(1, longest, n), np.arange(n + 1), 16, q_heads=16, kv_heads=2, dim=dim)
    check(gpu, b)


def test_one_unit_tiles_after_a_full_one(gpu):
    n = 301
    nodes = np.ones(n, int)
    nodes[0] = 140
    b = PrefixBatch(621, [2] * n, nodes, [128] * n, np.arange(n + 1), 8, q_heads=4, kv_heads=2, dim=64, dtype="bfloat16")
    check(gpu, b)
