"""The paged cache without a GPU: refusals of the C entry points, and the index arithmetic compiled for the host."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2504_08791_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    d = tmp_path_factory.mktemp("index")
    src = d / "index.cpp"
    src.write_text('''
#include "%s/paper_2504_08791_b200/csrc/paged_index.h"
extern "C" int64_t find(int layers, int pages, int shift, int heads, const int32_t* row, int64_t stride, int layer, int64_t slot) {
  return prima::find_slot({layers, pages, shift, heads}, row, stride, layer, slot);
}
using namespace prima;
extern "C" int64_t units(int heads, int group, int causal, int64_t capacity, int overhead, int tile, int ctx, int nodes) { return tree_units({heads, group, causal, capacity, overhead, tile}, ctx, nodes); }
extern "C" int64_t kv_end(int heads, int group, int causal, int64_t capacity, int tile, int ctx, int nodes, int rt) { return tree_kv_end({heads, group, causal, capacity, 0, tile}, ctx, nodes, rt); }
extern "C" int64_t share(int64_t units, int n, int c) { return tree_share_begin(tree_shares(units, n), c); }
extern "C" int cta_of(int64_t units, int n, int64_t u) { return tree_cta_of(tree_shares(units, n), u); }
extern "C" int small(int x, int d) { return small_div(x, small_inverse(d)); }
extern "C" void segment(int heads, int group, int causal, int64_t capacity, int overhead, int tile, int ctx, int nodes, int64_t u, int64_t end, int64_t* out) {
  const TreeShape t{heads, group, causal, capacity, overhead, tile};
  const TreeSegment s = tree_segment(t, ctx, nodes, tree_units(t, ctx, nodes), u, end);
  out[0] = s.head; out[1] = s.row_tile; out[2] = s.chunk0; out[3] = s.chunk1; out[4] = s.chunks; out[5] = s.places; out[6] = s.to_end;
}
''' % ROOT)
    lib = d / "index.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-shared", "-fPIC", str(src), "-o", str(lib)], check=True)
    L = ctypes.CDLL(str(lib))
    L.find.restype = ctypes.c_int64
    L.find.argtypes = [ctypes.c_int] * 4 + [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_int64]
    i32, i64 = ctypes.c_int, ctypes.c_int64
    L.units.restype = L.kv_end.restype = L.share.restype = i64
    L.units.argtypes = [i32, i32, i32, i64, i32, i32, i32, i32]
    L.kv_end.argtypes = [i32, i32, i32, i64, i32, i32, i32, i32]
    L.share.argtypes = [i64, i32, i32]
    L.cta_of.argtypes = [i64, i32, i64]
    L.segment.argtypes = [i32, i32, i32, i64, i32, i32, i32, i32, i64, i64, ctypes.c_void_p]
    return L


def test_slots_of_good_and_bad_tables(index):
    layers, pages, shift, heads = 3, 50, 4, 8
    row = np.array([7, 49, 0, -1, 50, -2 ** 31, 2 ** 31 - 1], np.int32)
    at = row.ctypes.data
    for layer in range(layers):
        for slot in range(-5, 16 * 7 + 40):
            got = index.find(layers, pages, shift, heads, at, 7, layer, slot)
            page = int(row[slot // 16]) if 0 <= slot < 112 else None
            if page is None:
                assert got == -2
            elif not 0 <= page < pages:
                assert got == -1
            else:
                assert got == ((layer * pages + page) * heads) * 16 + slot % 16
                assert got + (heads - 1) * 16 < layers * pages * heads * 16
    for slot in (2 ** 31, 2 ** 40, -2 ** 40, 2 ** 63 - 1, -2 ** 63):
        assert index.find(layers, pages, shift, heads, at, 7, 0, slot) == -2


def test_rows_of_a_large_cache_pass_32_bits_of_bytes(index):
    # 80 layers x 3000 pages x 8 heads x 64 positions: 1.2e8 rows of 256 bytes
    row = np.array([2999], np.int32)
    assert index.find(80, 3000, 6, 8, row.ctypes.data, 1, 79, 63) == ((79 * 3000 + 2999) * 8) * 64 + 63
    assert (((79 * 3000 + 2999) * 8) * 64 + 63) * 256 > 2 ** 32


def test_division_by_the_group(index):
    for d in range(1, 65):
        for x in range(256 + 64):
            assert index.small(x, d) == x // d


def test_shares_of_many_units(index):
    for total in (1, 147, 148, 149, 2 ** 31 - 1, 2 ** 31, 2 ** 40 + 12345):
        for cta in (0, 1, 77, 147):
            a, b = index.share(total, 148, cta), index.share(total, 148, cta + 1)
            assert b - a in (total // 148, total // 148 + 1)
            for u in {a, b - 1}:
                if a <= u < b:
                    assert index.cta_of(total, 148, u) == cta
        assert index.share(total, 148, 0) == 0 and index.share(total, 148, 148) == total


@pytest.mark.parametrize("seed", range(12))
def test_shares_of_tree_attention_cover_every_position_once(index, seed):
    """The segments of all CTAs, put together, are every unit of every (sequence, KV head, row tile), once, in order."""
    rs = np.random.RandomState(seed)
    n_seq, heads, group, causal, n_cta = int(rs.randint(1, 30)), int(rs.choice([1, 2, 8])), int(rs.choice([1, 3, 5, 8, 64])), int(seed % 2), int(rs.choice([1, 3, 148]))
    capacity, overhead, tile = int(rs.choice([512, 1 << 20])), int(rs.choice([0, 2, 5])), int(rs.choice([16, 32, 256]))
    ctx, nodes = rs.randint(0, 3000, n_seq), rs.choice([0, 1, 2, 16, 33, 64, 300], n_seq)
    want, places = [], 0
    for s in range(n_seq):
        for g in range(heads):
            for rt in range(-(-int(nodes[s]) * group // tile)):
                last_row = min(int(nodes[s]) * group, tile * (rt + 1)) - 1
                end = min(capacity, int(ctx[s]) + (last_row // group + 1 if causal else int(nodes[s])))
                got_end = index.kv_end(heads, group, causal, capacity, tile, int(ctx[s]), int(nodes[s]), rt)
                assert got_end == end
                want += [(s, g, rt, c, -(-end // 128)) for c in range(-(-end // 128))]
                places += overhead + -(-end // 128)
    per_seq = [heads * index.units(heads, group, causal, capacity, overhead, tile, int(c), int(n)) for c, n in zip(ctx, nodes)]
    total = sum(per_seq)
    assert total == places
    if not total:
        return
    got = []
    out = (ctypes.c_int64 * 7)()
    parts = {}      # CTAs that hold units of a (sequence, KV head, row tile)
    for cta in range(n_cta):
        u, end = index.share(total, n_cta, cta), index.share(total, n_cta, cta + 1)
        assert end - u in (total // n_cta, total // n_cta + 1)
        while u < end:
            assert index.cta_of(total, n_cta, u) == cta
            first, s = 0, 0
            while u >= first + per_seq[s]:
                first += per_seq[s]
                s += 1
            index.segment(heads, group, causal, capacity, overhead, tile, int(ctx[s]), int(nodes[s]), u - first, end - first, out)
            head, rt, c0, c1, chunks, n, to_end = out
            assert n > 0 and c1 >= c0
            got += [(s, head, rt, c, chunks) for c in range(c0, c1)]
            if c1 > c0:
                parts.setdefault((s, head, rt), []).append(cta)
                assert index.cta_of(total, n_cta, u + to_end - 1) >= cta
                parts[s, head, rt, "last"] = index.cta_of(total, n_cta, u + to_end - 1)
            u += n
    assert got == want
    # the parts of a whole lie in consecutive CTAs, up to the one that is named as the last
    for k, v in list(parts.items()):
        if len(k) == 3:
            assert v == list(range(v[0], v[-1] + 1)) and parts[(*k, "last")] == v[-1]


def test_refusals_need_no_gpu():
    build.build()
    L = binding.lib()
    h = ctypes.c_void_p()
    good = dict(n_layers=1, n_pages=4, page_size=16, n_kv_heads=2, head_dim=128, dtype=binding.DT_F16, rope_theta=1e4, rope_mode=0, device=0)

    def create(**change):
        c = binding.PagedConfig(*[{**good, **change}[n] for n, _ in binding.PagedConfig._fields_])
        return L.prima_paged_create(ctypes.byref(c), 4096, 8192, ctypes.byref(h))
    for change in (dict(n_layers=0), dict(n_pages=0), dict(page_size=4), dict(page_size=24), dict(page_size=65536), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(head_dim=96), dict(head_dim=256),
                   dict(dtype=binding.DT_F32), dict(dtype=7), dict(rope_theta=0.0), dict(rope_theta=float("inf")), dict(rope_theta=float("nan")), dict(rope_mode=2), dict(device=-1),
                   dict(n_pages=1 << 30), dict(n_layers=1 << 20, n_pages=1 << 20)):
        assert create(**change) == binding.ERR_ARG, change
        assert b"prima_paged_create" in L.prima_last_error(None)
    c = binding.PagedConfig(*[good[n] for n, _ in binding.PagedConfig._fields_])
    assert L.prima_paged_create(ctypes.byref(c), None, 8192, ctypes.byref(h)) == binding.ERR_ARG
    assert L.prima_paged_create(ctypes.byref(c), 4100, 8192, ctypes.byref(h)) == binding.ERR_ARG
    assert L.prima_paged_create(None, 4096, 8192, ctypes.byref(h)) == binding.ERR_ARG and not h.value
    b = binding.PagedBatchDesc(1, 1, 4096, 4096, 4096, 1, None, None, 0)
    ref = ctypes.byref(b)
    assert L.prima_paged_append(None, 0, ref, None, 4096, 4096, 0, 0, 0, 256, 256, None, None) == binding.ERR_ARG
    assert L.prima_paged_accept(None, ref, 4096, 4096, 1, None) == binding.ERR_ARG
    assert L.prima_paged_reorder(None, 1, 1, 1, 4096, 1, 4096, 4096, 4096, 4096, 4096, None) == binding.ERR_ARG
    assert L.prima_tree_attention(None, 0, ref, 4096, 2, 1.0, 4096, 1, None, 4096, 1 << 40, None) == binding.ERR_ARG
    assert L.prima_tree_attention_workspace(None, 1, 1, 1) == binding.ERR_ARG
    assert L.prima_paged_sync(None, None) == binding.ERR_ARG and L.prima_paged_destroy(None) == binding.OK
    select = [4096, 0, 1, 4, 100, 100, 4096, None, 0, 4, 4096, 4096, 4096, 4096, 1 << 40, None]
    for i, bad in ((0, None), (1, 3), (2, 0), (3, 0), (3, 65), (4, 0), (5, 99), (6, None), (9, 0), (9, 65), (10, None), (11, None), (12, None), (13, None), (13, 4224), (14, 8)):
        args = list(select)
        args[i] = bad
        assert L.prima_beam_select(*args) == binding.ERR_ARG, (i, bad)
    args = list(select)
    args[7], args[8] = 4096, 100      # an end token outside the vocabulary
    assert L.prima_beam_select(*args) == binding.ERR_ARG
    assert L.prima_beam_select_workspace(1, 64, 1 << 26, 4) == binding.ERR_ARG
    assert L.prima_beam_select_workspace(16, 8, 152064, 8) > 0


def test_vocabularies_up_to_32_bits():
    """Words are numbered in 32 bits up to the end of the last slice of 8192: longer rows are refused as arguments."""
    build.build()
    L = binding.lib()
    longest = 2 ** 31 - 8192
    assert L.prima_beam_select_workspace(1, 1, longest, 4) > 0
    for vocab in (longest + 1, 2 ** 31 - 2048, 2 ** 31 - 1):
        assert L.prima_beam_select_workspace(1, 1, vocab, 4) == binding.ERR_ARG, vocab
        assert L.prima_beam_select(4096, binding.DT_F16, 1, 1, vocab, vocab, 4096, None, 0, 4, 4096, 4096, 4096, 4096, 1 << 40, None) == binding.ERR_ARG
        assert b"vocab" in L.prima_last_error(None)


class Stand:
    """What the binding looks at in a tensor."""

    def __init__(self, dtype, *shape):
        self.dtype, self.shape, self.device, self.is_cuda = dtype, shape, "cuda:0", True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096 if self.numel() else 0      # torch: no address without elements


def test_a_mask_without_words_is_refused():
    """It has no address, and a batch without a mask is a causal one."""
    import torch
    i32 = torch.int32
    table, begin, ctx = Stand(i32, 2, 5), Stand(i32, 3), Stand(i32, 2)
    assert binding.PagedBatch(table, begin, ctx, 4, mask=Stand(torch.int64, 4, 1)).desc.mask_words == 1
    assert binding.PagedBatch(table, begin, ctx, 4).desc.mask is None
    with pytest.raises(ValueError):
        binding.PagedBatch(table, begin, ctx, 4, mask=Stand(torch.int64, 4, 0))
