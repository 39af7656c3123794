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
    assert axes.n_axes == 3 and axes.pairs == 32 and axes.axis[16] == binding.AXIS_NONE and axes.rank[31] == 31
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
