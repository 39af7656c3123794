"""Kernels of a bounded cache right behind one another, each reading what the one in front has just written (lengths of an
eviction in place, queries of an append, log-sum-exps of an attention): the bits of the same calls with a pause between them."""
import numpy as np
import pytest

from tests._prefix import PrefixBatch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401
from tests.test_gpu_prefix_attention import prefix_on_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 24], ids=["few rows", "many rows"])
@pytest.mark.parametrize("seqs", [3, 70])
def test_calls_without_a_pause_give_the_bits_of_calls_with_one(gpu, seqs, rows):
    torch, binding = gpu
    rs = np.random.RandomState(seqs)
    ctx = rs.randint(100, 160, seqs)
    b = PrefixBatch(640, ctx, [rows] * seqs, [200], [0, seqs], 16, q_heads=4, kv_heads=2, dim=64)
    slots, n = 200, b.n_tok
    x = [on_gpu(torch, rs.standard_normal((n, 8, 64)).astype(np.float32)) for _ in range(8)]
    keeps = [on_gpu(torch, np.full(seqs, 95 - 11 * i, np.int32)) for i in range(8)]
    gain, table, prefix = torch.ones(64, device="cuda"), on_gpu(torch, b.table), prefix_on_gpu(gpu, b)
    w0 = on_gpu(torch, np.exp(rs.standard_normal((1, seqs, 2, slots))).astype(np.float32))
    row_begin, pos = on_gpu(torch, b.row_begin), on_gpu(torch, np.arange(n, dtype=np.int32) + 1000)
    scratch = binding.PagedCache(*cache_on_gpu(gpu, b)[:2])
    batch = batch_on_gpu(gpu, b)
    workspace, room = scratch.prefix_attention_workspace(batch, prefix, 4), scratch.evict_workspace(seqs, slots)

    def state():
        k, v, pool = cache_on_gpu(gpu, b)
        length = on_gpu(torch, b.ctx)
        return {"k": k, "v": v, "pool": pool, "length": length, "w": w0.clone(), "born": torch.arange(slots, dtype=torch.int32, device="cuda").repeat(1, seqs, 2, 1),
                "q": torch.zeros((8, n, 4, 64), dtype=torch.float16, device="cuda"), "out": torch.zeros((8, n, 4, 64), dtype=torch.float16, device="cuda"),
                "lse": torch.zeros((8, n, 4), device="cuda"), "batch": binding.PagedBatch(table, row_begin, length, n, pos=pos)}

    def steps(s, pause):
        pool = s["pool"]
        for i in range(8):
            pool.evict(table, s["length"], s["w"], s["born"], keeps[i], s["length"], workspace=room)
            pause()
            pool.append_norm(0, s["batch"], x[i][:, :4], x[i][:, 4:6], x[i][:, 6:], s["q"][i], q_gain=gain, k_gain=gain)
            pause()
            pool.prefix_attention(0, s["batch"], prefix, s["q"][i], s["out"][i], lse=s["lse"][i], workspace=workspace)
            pause()
            pool.attention_weights(0, s["batch"], s["q"][i], s["lse"][i], s["w"][0], weight_in=s["w"][0], born=s["born"][0])
            pause()
    want = state()
    steps(want, torch.cuda.synchronize)
    assert want["length"].tolist() == [18] * seqs and not torch.isnan(want["out"]).any()
    got = state()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(got, lambda: None)
    for _ in range(20):
        fresh = state()
        for name in ("k", "v", "length", "w", "born"):
            got[name].copy_(fresh[name])
        for name in ("q", "out", "lse"):
            got[name].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("k", "v", "length", "w", "born", "q", "out", "lse"):
            assert torch.equal(got[name], want[name]), name
    got["pool"].sync()
    want["pool"].sync()
