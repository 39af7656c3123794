"""Beam selection against a selection over all candidates in 64 bits."""
import numpy as np
import pytest

from tests import _paged
from tests.test_gpu_paged import gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


def run(gpu, logits, cum, keep, finished=None, end=0, dtype="float32", offset=0, row_pad=0, stream=None):
    torch, binding = gpu
    n_req, n_beams, vocab = logits.shape
    flat = torch.full((offset + n_req * n_beams * (vocab + row_pad),), 50.0, dtype=getattr(torch, dtype), device="cuda")
    dev = flat[offset:].view(n_req, n_beams, vocab + row_pad)[..., :vocab]
    dev.copy_(on_gpu(torch, logits))
    score = torch.full((n_req, keep), 7.0, device="cuda")
    parent, token = torch.full((n_req, keep), 7, dtype=torch.int32, device="cuda"), torch.full((n_req, keep), 7, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    binding.prima_beam_select(dev, on_gpu(torch, cum), score, parent, token, finished=None if finished is None else on_gpu(torch, finished), end_token=end, stream=stream)
    torch.cuda.synchronize()
    return score.cpu().numpy(), parent.cpu().numpy(), token.cpu().numpy()


def check(gpu, logits, cum, keep, finished=None, end=0, dtype="float32", **more):
    logits = _paged.rounded(logits.astype(np.float32), dtype)
    got = run(gpu, logits, cum, keep, finished, end, dtype, **more)
    want = _paged.beam_select(logits, cum, keep, finished, end)
    # score: 2^-24 for its rounding; log of a sum whose terms are off by 2^-21 at most
    fine = np.isfinite(want[0])
    assert np.array_equal(np.isneginf(got[0]), ~fine)
    assert np.all(np.abs(got[0][fine] - want[0][fine]) <= 2.0 ** -24 * np.abs(want[0][fine]) + 2.0 ** -20)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2])
    return got


def some(seed, n_req, n_beams, vocab, spread=3.0):
    rs = np.random.RandomState(seed)
    return rs.standard_normal((n_req, n_beams, vocab)) * spread, -rs.gamma(3.0, 1.0, (n_req, n_beams)).astype(np.float32), rs


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("n_req,n_beams,vocab,keep", [(1, 1, 1, 1), (1, 1, 5, 8), (2, 3, 31, 3), (1, 4, 32000, 4), (3, 8, 2049, 16), (2, 5, 128259, 5), (1, 64, 700, 64),
                                                      (4, 2, 8192, 1), (1, 7, 8193, 33), (40, 16, 1000, 16)])
def test_shapes(gpu, dtype, n_req, n_beams, vocab, keep):
    logits, cum, _ = some(1, n_req, n_beams, vocab)
    check(gpu, logits, cum, keep, dtype=dtype)


@pytest.mark.parametrize("offset,row_pad", [(1, 0), (0, 1), (3, 5), (4, 4), (0, 8)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_unaligned_rows_give_the_same_bits(gpu, offset, row_pad, dtype):
    logits, cum, _ = some(2, 2, 3, 4100)
    logits = _paged.rounded(logits.astype(np.float32), dtype)
    a, b = run(gpu, logits, cum, 6, dtype=dtype), check(gpu, logits, cum, 6, dtype=dtype, offset=offset, row_pad=row_pad)
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_ties_go_to_the_lowest_index(gpu):
    for vocab in (64, 9000, 40000):
        logits = np.zeros((2, 4, vocab))
        check(gpu, logits, np.zeros((2, 4), np.float32), 10)                      # all candidates equal, across beams too
        logits[:, :, 17::13] = 1.0
        check(gpu, logits, np.zeros((2, 4), np.float32), 64)
        logits[:, 1:] = logits[:, :1]
        check(gpu, logits, np.full((2, 4), -2.5, np.float32), 7, dtype="bfloat16")
    # equal rows at the first step: only beam 0 is alive
    cum = np.full((2, 4), -np.inf, np.float32)
    cum[:, 0] = 0
    check(gpu, logits, cum, 4)


def test_many_equal_scores_in_every_beam(gpu):
    """More candidates at the bound than the second kernel keeps."""
    logits = np.zeros((1, 64, 4096))
    check(gpu, logits, np.zeros((1, 64), np.float32), 64)
    logits[0, 5, 100] = 2.0
    check(gpu, logits, np.zeros((1, 64), np.float32), 64)


def test_finished_beams_keep_their_score(gpu):
    logits, cum, rs = some(4, 6, 8, 5000)
    finished = (rs.rand(6, 8) < 0.4).astype(np.uint8)
    finished[0], finished[1] = 1, 0
    check(gpu, logits, cum, 8, finished, end=4999)
    check(gpu, logits, cum, 64, finished, end=0)
    cum[0, 2] = -np.inf
    check(gpu, logits, cum, 8, finished, end=17)
    logits[finished.astype(bool)] = np.nan      # what a finished beam's row holds does not matter
    check(gpu, logits, cum, 8, finished, end=17)


def test_masked_words(gpu):
    logits, cum, rs = some(5, 2, 4, 3001)
    logits[:, :, rs.rand(3001) < 0.9] = -np.inf
    check(gpu, logits, cum, 8)
    logits[0, 1] = -np.inf                      # a row with nothing left
    logits[1, :, 5:] = -np.inf                  # fewer candidates than places
    check(gpu, logits, cum, 32)
    logits[0, 2, ::2] = np.nan
    check(gpu, logits, cum, 16)
    logits[:] = -np.inf
    got = check(gpu, logits, cum, 3)
    assert np.all(got[1] == 0) and np.all(got[2] == -1)
    low = np.full((1, 2, 2500), np.finfo(np.float32).min)
    check(gpu, low, np.zeros((1, 2), np.float32), 5)      # the type's lowest value is a value
    low[0, 0, 77] = 0
    check(gpu, low, np.zeros((1, 2), np.float32), 5)
    check(gpu, np.full((1, 2, 300), -65504.0), np.zeros((1, 2), np.float32), 5, dtype="float16")


def test_infinite_and_large_logits(gpu):
    logits, cum, _ = some(6, 1, 3, 2600)
    logits[0, 0, 9] = logits[0, 0, 2000] = np.inf         # the largest finite value, twice
    got = run(gpu, logits.astype(np.float32), cum, 4)
    want = _paged.beam_select(logits.astype(np.float32), cum, 4)
    assert np.array_equal(got[1], want[1]) and np.array_equal(got[2], want[2]) and np.allclose(got[0], want[0], rtol=1e-6, atol=1e-6)
    logits = np.random.RandomState(0).standard_normal((1, 3, 2600)) * 1e4
    check(gpu, logits, cum, 6)


def test_dead_beams(gpu):
    logits, cum, _ = some(7, 3, 4, 900)
    cum[0] = -np.inf
    cum[1, 1:] = np.nan
    check(gpu, logits, np.where(np.isnan(cum), -np.inf, cum).astype(np.float32), 6)
    a = run(gpu, logits.astype(np.float32), cum, 6)
    b = run(gpu, logits.astype(np.float32), np.where(np.isnan(cum), -np.inf, cum).astype(np.float32), 6)
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_captured_and_on_other_streams(gpu):
    torch, binding = gpu
    logits, cum, _ = some(8, 2, 4, 12000)
    want = run(gpu, logits.astype(np.float32), cum, 4)
    got = run(gpu, logits.astype(np.float32), cum, 4, stream=torch.cuda.Stream())
    assert all(np.array_equal(x, y) for x, y in zip(got, want))
    dev, dc = on_gpu(torch, logits.astype(np.float32)), on_gpu(torch, cum)
    outs = torch.zeros((2, 4), device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.prima_beam_select(dev, dc, *outs)
    for _ in range(3):
        dev.copy_(torch.flip(dev, (0,)))
        dc.copy_(torch.flip(dc, (0,)))
        g.replay()
    torch.cuda.synchronize()
    assert all(np.array_equal(x.cpu().numpy(), y[::-1]) for x, y in zip(outs, want))
    del g


def test_argument_errors(gpu):
    torch, binding = gpu
    x = torch.zeros((2, 3, 50), device="cuda")
    cum = torch.zeros((2, 3), device="cuda")

    def outs(k, r=2):
        return torch.zeros((r, k), device="cuda"), torch.zeros((r, k), dtype=torch.int32, device="cuda"), torch.zeros((r, k), dtype=torch.int32, device="cuda")
    done = torch.zeros((2, 3), dtype=torch.uint8, device="cuda")
    ws = binding.prima_beam_select_workspace(2, 3, 50, 4)
    for call in (lambda: binding.prima_beam_select(x, cum, *outs(65)), lambda: binding.prima_beam_select(x.double(), cum, *outs(4)), lambda: binding.prima_beam_select(x, cum[:1], *outs(4)),
                 lambda: binding.prima_beam_select(x, cum, *outs(4, 1)), lambda: binding.prima_beam_select(x, cum, *outs(4), finished=done), lambda: binding.prima_beam_select(x.transpose(0, 1), cum, *outs(4)),
                 lambda: binding.prima_beam_select(x, cum, *outs(4), finished=done, end_token=50), lambda: binding.prima_beam_select(x, cum, *outs(4), finished=done.bool(), end_token=1),
                 lambda: binding.prima_beam_select(x, cum, *outs(4), workspace=ws[:16]), lambda: binding.prima_beam_select(x, cum, *outs(4), workspace=ws[1:]),
                 lambda: binding.prima_beam_select(torch.zeros((1, 65, 5), device="cuda"), torch.zeros((1, 65), device="cuda"), *outs(4, 1)), lambda: binding.prima_beam_select(x.cpu(), cum, *outs(4)),
                 lambda: binding.prima_beam_select_workspace(0, 1, 5, 1), lambda: binding.prima_beam_select_workspace(1, 64, 1 << 26, 1)):
        with pytest.raises((ValueError, binding.PrimaError)):
            call()


@pytest.mark.parametrize("words", [1, 3, 8, 40, 511, 513, 1791])
@pytest.mark.parametrize("dtype,keep", [("float32", 8), ("bfloat16", 8), ("float32", 40), ("float16", 64)])
def test_short_last_slices(gpu, words, dtype, keep):
    """A row that ends a few words into a slice, the best of it among them."""
    logits, cum, _ = some(11, 1, 2, 2048 * 3 + words)
    logits[:, :, -words:] += 6.0
    check(gpu, logits, cum, keep, dtype=dtype)


@pytest.mark.parametrize("n_beams,keep", [(8, 8), (5, 3), (16, 16), (3, 64)])
def test_one_beam_holds_the_best(gpu, n_beams, keep):
    logits, cum, _ = some(12, 2, n_beams, 40000)
    cum[:] -= 100.0
    cum[0, n_beams - 1] = cum[1, 0] = -1.0
    check(gpu, logits, cum, keep)


@pytest.mark.parametrize("n_req,n_beams,vocab,dtype", [(16, 8, 152064, "float32"), (1, 64, 152064, "bfloat16")])
def test_the_longest_list_takes_no_search_word_by_word(gpu, n_req, n_beams, vocab, dtype):
    """64 kept continuations of logits in no order: as many CTAs as these would meet a list that runs over in nearly every
    call, and each would then go through its words 64 times (15 times the time of 63 kept ones)."""
    torch, binding = gpu
    torch.manual_seed(5)
    x = (torch.randn((n_req, n_beams, vocab), device="cuda") * 2.2).to(getattr(torch, dtype))
    cum = torch.randn((n_req, n_beams), device="cuda")
    times = {}
    for keep in (63, 64):
        out = torch.zeros((n_req, keep), device="cuda"), torch.zeros((n_req, keep), dtype=torch.int32, device="cuda"), torch.zeros((n_req, keep), dtype=torch.int32, device="cuda")
        events = [(torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)) for _ in range(9)]
        for a, b in events:
            a.record()
            binding.prima_beam_select(x, cum, *out)
            b.record()
        torch.cuda.synchronize()
        times[keep] = sorted(a.elapsed_time(b) for a, b in events)[4]
        for r in range(n_req):      # two candidates that change places differ by their errors, 2^-20 each (see check)
            score = cum[r].double()[:, None] + torch.log_softmax(x[r].double(), 1)
            want = torch.topk(score.flatten(), keep).values
            got = score[out[1][r].long(), out[2][r].long()]
            assert torch.all((got - want).abs() <= 2.0 ** -19)
            assert torch.unique(out[1][r].long() * vocab + out[2][r].long()).numel() == keep
    assert times[64] < 4 * times[63], times
