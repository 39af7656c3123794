"""Append with norms where a warp has a row to itself, on both sides of the rule (three rows per SM), in graphs and on other streams."""
import numpy as np
import pytest

from tests._paged import Batch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401
from tests.test_gpu_paged_norm import THETA, check, three

pytestmark = pytest.mark.gpu


def batch_of(gpu, rows, seed, dim, dtype="float16", **kw):
    """Three sequences with `rows` rows in all, one of them a single token; padding comes on top of `rows` where it is asked for."""
    return Batch(seed, ctx=[0, 30, 7], nodes=[rows - 1 - rows // 3, 1, rows // 3], page=16, kv_heads=2, q_heads=4, dim=dim, dtype=dtype, **kw)


def rule(gpu):
    return 3 * gpu[0].cuda.get_device_properties(0).multi_processor_count


@pytest.mark.parametrize("dtype,src", [("float16", "float32"), ("float16", "float16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("dim,mode", [(128, 0), (64, 1), (128, 1), (64, 0)])
@pytest.mark.parametrize("gains", ["shared", "each"])
def test_types_and_layouts(gpu, dtype, src, dim, mode, gains):
    b = batch_of(gpu, rule(gpu) + 7, 520, dim, dtype, pad=2, layers=2)
    check(gpu, b, src, mode, gains, axes=([i % 3 for i in range(dim // 2)],), positions=three(b.rs, b.n_tok), layer=1)


@pytest.mark.parametrize("offset,gain_offset", [(0, 1), (1, 0), (8, 4)])
@pytest.mark.parametrize("src", ["float32", "float16"])
def test_unaligned_sources_and_gains(gpu, offset, gain_offset, src):
    check(gpu, batch_of(gpu, rule(gpu) + 3, 521, 128), src, 0, "each", offset=offset, gain_offset=gain_offset)


@pytest.mark.parametrize("more", [-1, 0, 1, 2])
@pytest.mark.parametrize("gains", ["q", "k", "none"])
def test_both_sides_of_the_rule(gpu, more, gains):
    check(gpu, batch_of(gpu, rule(gpu) + more, 522, 64), "float16", 0, gains)


def test_no_queries(gpu):
    check(gpu, batch_of(gpu, rule(gpu) + 5, 523, 128), "float16", 1, with_q=False)


@pytest.mark.parametrize("rows", [5, 500])
def test_without_gains_and_axes_it_is_the_plain_append(gpu, rows):
    torch, binding = gpu
    b = batch_of(gpu, rows, 524, 128)
    for mode in (0, 1):
        x = torch.randn((b.n_tok, 8, 128), device="cuda").half()
        seen = []
        for call in ("append", "append_norm"):
            k, v, pool = cache_on_gpu(gpu, b, THETA, mode)
            q = torch.empty((b.n_tok, 4, 128), dtype=torch.float16, device="cuda")
            getattr(pool, call)(0, batch_on_gpu(gpu, b), x[:, :4], x[:, 4:6], x[:, 6:], q)
            pool.sync()
            seen.append((q, k, v))
        assert all(torch.equal(a, c) for a, c in zip(*seen))


@pytest.mark.parametrize("rows", [5, 500])
def test_graphs_and_streams(gpu, rows):
    """Captured and replayed with other lengths and other rows; two calls at once on streams of their own."""
    torch, binding = gpu
    b = batch_of(gpu, rows, 525, 64)
    gain, pos = torch.rand((4, 64), device="cuda") + 0.5, on_gpu(torch, three(b.rs, b.n_tok))
    axes = binding.RopeAxes([i % 3 for i in range(32)])
    x = torch.randn((b.n_tok, 8, 64), device="cuda")
    ctx, row_begin, table = on_gpu(torch, b.ctx), on_gpu(torch, b.row_begin), on_gpu(torch, b.table)
    batch = binding.PagedBatch(table, row_begin, ctx, b.n_tok)

    def call(c, q, stream=None):
        c[2].append_norm(0, batch, x[:, :4], x[:, 4:6], x[:, 6:], q, q_gain=gain, k_gain=gain[0], positions=pos, axes=axes, stream=stream)
    caches = [cache_on_gpu(gpu, b, THETA) for _ in range(4)]
    out = [torch.zeros((b.n_tok, 4, 64), dtype=torch.float16, device="cuda") for _ in range(4)]
    call(caches[0], out[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(caches[1], out[1])
    for shift in (0, 2, 5):
        x.copy_(torch.randn_like(x))
        pos.add_(17)
        ctx.copy_(on_gpu(torch, np.maximum(b.ctx - shift, 0)))
        fresh = cache_on_gpu(gpu, b, THETA)
        for c in caches:
            c[0].copy_(fresh[0])
            c[1].copy_(fresh[1])
        for o in out:
            o.zero_()
        torch.cuda.synchronize()
        call(caches[0], out[0])
        graph.replay()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        torch.cuda.synchronize()
        for i in range(2):
            call(caches[2 + i], out[2 + i], streams[i])
        torch.cuda.synchronize()
        for i in range(1, 4):
            assert torch.equal(out[i], out[0]) and torch.equal(caches[i][0], caches[0][0]) and torch.equal(caches[i][1], caches[0][1])
        assert out[0].any()
    for c in caches:
        c[2].sync()
