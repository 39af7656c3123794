"""Operators of long prompts and bounded caches: what needs no GPU (refusals, their 64-bit definitions)."""
import ctypes

import numpy as np
import pytest

from paper_2504_08791_b200 import binding, build
from tests import _prefix
from tests.test_paged_cpu import Stand


def test_refusals_need_no_gpu():
    build.build()
    L = binding.lib()
    ref = ctypes.byref(binding.PagedBatchDesc(1, 1, 4096, 4096, 4096, 1, None, None, 0))
    norm, prefix = ctypes.byref(binding.HeadNormDesc(eps=1e-6, n_axes=1)), ctypes.byref(binding.PrefixDesc(1, 4096, 4096, 4096, 1))
    assert L.prima_paged_append_norm(None, 0, ref, None, 4096, 4096, 0, 0, 0, 256, 256, norm, None, None) == binding.ERR_ARG
    assert L.prima_prefix_attention(None, 0, ref, prefix, 4096, 2, 1.0, 4096, 1, None, 4096, 1 << 40, None) == binding.ERR_ARG
    assert L.prima_paged_weights(None, 0, ref, 4096, 2, 1.0, 4096, None, 4096, None, 8, 1.0, None) == binding.ERR_ARG
    assert L.prima_paged_evict(None, 1, 4096, 1, 4096, 4096, 4096, 8, 4096, 0, None, 4096, 4096, 4096, 4096, 1 << 40, None) == binding.ERR_ARG
    assert b"prima_paged_evict" in L.prima_last_error(None)
    assert L.prima_prefix_attention_workspace(None, 1, 1, 1) == binding.ERR_ARG
    assert L.prima_paged_evict_workspace(None, 1, 1) == binding.ERR_ARG


def test_structures_are_those_of_the_header():
    """Sizes and offsets as a C compiler lays them out."""
    assert ctypes.sizeof(binding.HeadNormDesc) == 48 + 128 and binding.HeadNormDesc.positions.offset == 40 and binding.HeadNormDesc.axis.offset == 48
    assert ctypes.sizeof(binding.PrefixDesc) == 40 and binding.PrefixDesc.seq_begin.offset == 8


def test_axes_and_prefixes_are_checked():
    import torch
    i32 = torch.int32
    axes = binding.RopeAxes([0] * 8 + [2] * 8 + [-1] * 16)
    assert axes.n_axes == 3 and axes.pairs == 32 and axes.desc.axis[16] == binding.AXIS_NONE and axes.desc.rank[31] == 31
    assert binding.RopeAxes([-1] * 64).n_axes == 1
    for axis, rank in (([0] * 33, None), ([0] * 32, [0] * 31), ([0] * 32, [0] * 31 + [32]), ([4] * 32, None), ([-2] * 32, None)):
        with pytest.raises(ValueError):
            binding.RopeAxes(axis, rank)
    assert binding.PrefixBatch(Stand(i32, 2, 5), Stand(i32, 2), Stand(i32, 3)).desc.table_stride == 5
    for bad in ((Stand(i32, 3, 5), Stand(i32, 2), Stand(i32, 3)), (Stand(i32, 2, 5), Stand(i32, 2), Stand(i32, 2)), (Stand(i32, 10), Stand(i32, 2), Stand(i32, 3)),
                (Stand(i32, 2, 5), Stand(torch.int64, 2), Stand(i32, 3))):
        with pytest.raises(ValueError):
            binding.PrefixBatch(*bad)


def test_choices_of_an_eviction():
    w = np.array([1, 5, np.nan, 3, 3, 0, -np.inf, 9], np.float32)
    born = np.arange(8)
    kept, source = _prefix.choose(w, born, 8, 3, 0, None)
    assert kept.tolist() == [1, 3, 7] and source.tolist() == [3, 1, 7]      # of equal ones the lower slot; the others move up
    assert _prefix.choose(w, born, 8, 3, 1, 6)[0].tolist() == [0, 6, 7]
    assert _prefix.choose(w, born, 8, 2, 1, 6)[0].tolist() == [0, 6]        # protected entries are equal among themselves
    assert _prefix.choose(w, born, 8, 7, 0, None)[0].tolist() == [0, 1, 3, 4, 5, 6, 7]
    assert _prefix.choose(w, born, 2, 7, 0, None)[1].tolist() == [0, 1]


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    """The index arithmetic of the shared prefixes, compiled for the host."""
    import os
    import subprocess
    at = tmp_path_factory.mktemp("prefix_index")
    src, out = str(at / "x.cpp"), str(at / "x.so")
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2504_08791_b200", "csrc", "paged_index.h")
    with open(src, "w") as f:
        f.write(f'''#include "{header}"
using namespace prima;
extern "C" {{
long long places(int heads, long long cap, int over, long long rows, int len) {{ PrefixShape t{{heads, cap, over}}; return prefix_places(t, rows, prefix_units(t, len)); }}
long long units(int heads, long long cap, int over, int len) {{ PrefixShape t{{heads, cap, over}}; return prefix_units(t, len); }}
long long own_places_(int rows, long long limit) {{ return own_places(rows, limit); }}
void own(long long limit, long long per_head, long long u, long long end, long long* out) {{
  const OwnSegment s = own_segment(limit, per_head, u, end);
  out[0] = s.head; out[1] = s.tile; out[2] = s.step0; out[3] = s.step1; out[4] = s.places; out[5] = s.last;
}}
int workers(long long p, long long o, int cost, int n) {{ return prefix_workers(p, o, cost, n); }}
long long begin(long long total, int n, int c) {{ return tree_share_begin(tree_shares(total, n), c); }}
int owner(long long total, int n, long long u) {{ return tree_cta_of(tree_shares(total, n), u); }}
void segment(int heads, long long cap, int over, long long rows, int len, long long u, long long end, long long* out) {{
  PrefixShape t{{heads, cap, over}};
  const long long n = prefix_units(t, len);
  const PrefixSegment s = prefix_segment(t, rows, n, prefix_places(t, rows, n), u, end);
  out[0] = s.head; out[1] = s.row_tile; out[2] = s.unit0; out[3] = s.unit1; out[4] = s.places; out[5] = s.first; out[6] = s.last;
}}
}}''')
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-std=c++17", "-o", out, src], check=True)
    L = ctypes.CDLL(out)
    i64, i32 = ctypes.c_longlong, ctypes.c_int
    L.places.argtypes, L.places.restype = [i32, i64, i32, i64, i32], i64
    L.units.argtypes, L.units.restype = [i32, i64, i32, i32], i64
    L.own_places = L.own_places_
    L.own_places.argtypes, L.own_places.restype = [i32, i64], i64
    L.own.argtypes = [i64, i64, i64, i64, ctypes.POINTER(i64)]
    L.workers.argtypes = [i64, i64, i32, i32]
    L.begin.argtypes, L.begin.restype = [i64, i32, i32], i64
    L.owner.argtypes = [i64, i32, i64]
    L.segment.argtypes = [i32, i64, i32, i64, i32, i64, i64, ctypes.POINTER(i64)]
    return L


@pytest.mark.parametrize("seed", range(40))
def test_shares_of_the_prefixes_cover_every_unit_once(index, seed):
    """Every unit of every (prefix, KV head, tile) belongs to one worker; the workers of a tile are consecutive and each has a
    unit; the first and the last are those that the places name."""
    rs = np.random.RandomState(seed)
    heads, over, n_cta = int(rs.randint(1, 9)), 4, int(rs.choice([2, 3, 7, 148]))
    n_prefix = int(rs.choice([1, 1, 2, 5]))
    rows = rs.choice([0, 1, 16, 127, 128, 129, 255, 256, 257, 384, 385, 512, 1000], n_prefix)
    length = rs.choice([0, 1, 127, 128, 129, 500, 3000, 40000], n_prefix)
    cap = int(rs.choice([100, 1024, 1 << 20]))
    per_head = [index.places(heads, cap, over, int(r), int(n)) for r, n in zip(rows, length)]
    total = sum(per_head) * heads
    own = int(rs.choice([0, 5, 1000]))
    n = index.workers(total, own, 128, n_cta)
    if total == 0:
        assert n == 0
        return
    assert 1 <= n <= (n_cta if own == 0 else n_cta - 1) and (n == 1 or total // n >= 2)
    front = np.concatenate([[0], np.cumsum([p * heads for p in per_head])])
    seen, out = {}, (ctypes.c_longlong * 7)()
    for c in range(n):
        u, end = index.begin(total, n, c), index.begin(total, n, c + 1)
        while u < end:
            p = int(np.searchsorted(front, u, side="right")) - 1
            while per_head[p] == 0:
                p += 1
            index.segment(heads, cap, over, int(rows[p]), int(length[p]), u - int(front[p]), end - int(front[p]), out)
            head, tile, unit0, unit1, places, first, last = list(out)
            assert 0 <= head < heads and 0 <= tile <= (rows[p] - 1) // 256 and places > 0 and 0 <= unit0 <= unit1
            if unit1 > unit0:
                seen.setdefault((p, head, tile), []).append((c, unit0, unit1))
                if unit0 == 0:
                    assert index.owner(total, n, first + int(front[p])) == c
                last_owner = index.owner(total, n, last + int(front[p]))
                assert last_owner >= c and (unit1 == index.units(heads, cap, over, int(length[p]))) == (last_owner == c)
            u += places
        assert u == end
    for p in range(n_prefix):
        units = index.units(heads, cap, over, int(length[p]))
        for head in range(heads):
            for tile in range(-(-int(rows[p]) // 256) if units else 0):
                parts = seen.pop((p, head, tile))
                assert [x[1] for x in parts] == [0] + [x[2] for x in parts[:-1]] and parts[-1][2] == units
                assert [x[0] for x in parts] == list(range(parts[0][0], parts[0][0] + len(parts)))
    assert not seen


def test_workers_of_prefixes_and_own_positions(index):
    assert index.workers(0, 100, 128, 148) == 0 and index.workers(100, 0, 128, 148) == 50 and index.workers(10 ** 6, 0, 128, 148) == 148
    assert index.workers(1, 10 ** 9, 128, 148) == 1 and index.workers(10 ** 9, 1, 128, 148) == 147
    assert index.workers(1000, 500, 128, 148) == 74 and index.workers(1 << 50, 1 << 50, 64, 148) == 74


@pytest.mark.parametrize("seed", range(25))
def test_shares_of_the_own_positions_cover_every_step_once(index, seed):
    rs = np.random.RandomState(seed)
    heads, n = int(rs.randint(1, 9)), int(rs.choice([1, 8, 9, 800]))
    rows = rs.choice([0, 1, 5, 8, 16, 17, 33, 64], 12)
    limit = rs.choice([1, 15, 16, 17, 128, 700, 3000], 12)
    per_head = [index.own_places(int(r), int(m)) for r, m in zip(rows, limit)]
    total = sum(per_head) * heads
    if total == 0:
        return
    front = np.concatenate([[0], np.cumsum([p * heads for p in per_head])])
    seen, out = {}, (ctypes.c_longlong * 6)()
    for c in range(n):
        u, end = index.begin(total, n, c), index.begin(total, n, c + 1)
        while u < end:
            s = int(np.searchsorted(front, u, side="right")) - 1
            index.own(int(limit[s]), per_head[s], u - int(front[s]), end - int(front[s]), out)
            head, tile, step0, step1, places, last = list(out)
            assert 0 <= head < heads and 0 <= tile < -(-int(rows[s]) // 16) and places > 0 and 0 <= step0 <= step1
            if step1 > step0:
                seen.setdefault((s, head, tile), []).append((c, step0, step1))
                owner = index.owner(total, n, last + int(front[s]))
                assert owner >= c and (step1 == -(-int(limit[s]) // 16)) == (owner == c)
            u += places
        assert u == end
    for s in range(12):
        for head in range(heads):
            for tile in range(-(-int(rows[s]) // 16)):
                parts = seen.pop((s, head, tile))
                assert [x[1] for x in parts] == [0] + [x[2] for x in parts[:-1]] and parts[-1][2] == -(-int(limit[s]) // 16)
                assert [x[0] for x in parts] == list(range(parts[0][0], parts[0][0] + len(parts)))
    assert not seen
