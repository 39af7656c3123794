"""Norm of query and key heads, rotation on several axes and append in one pass, against 64 bits."""
import numpy as np
import pytest

from tests import _paged, _prefix
from tests._paged import Batch
from tests.test_gpu_paged import batch_on_gpu, cache_on_gpu, gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

THETA = 5e5


def check(gpu, b, src, mode=0, gains="shared", axes=None, positions=None, pos=None, eps=1e-6, layer=0, with_q=True, offset=0, x=None, size=3.0, gain_offset=0):
    torch, binding = gpu
    k, v, pool = cache_on_gpu(gpu, b, THETA, mode)
    H, G, D = b.q_heads, b.kv_heads, b.dim
    if x is None:
        x = b.rs.standard_normal((b.n_tok, H + 2 * G, D)).astype(np.float32) * size
    x = _paged.rounded(x, src)
    flat = torch.empty(offset + x.size, dtype=getattr(torch, src), device="cuda")
    dx = flat[offset:].view(b.n_tok, H + 2 * G, D)
    dx.copy_(on_gpu(torch, x))
    gain = {n: (1 + 0.3 * b.rs.standard_normal((h, D))).astype(np.float32) if gains == "each" else np.broadcast_to((1 + 0.3 * b.rs.standard_normal(D)).astype(np.float32), (h, D))
            if gains == "shared" or gains == n else None for n, h in (("q", H), ("k", G))}

    def gain_on_gpu(n):
        if gain[n] is None:
            return None
        a = gain[n] if gains == "each" else gain[n][0].copy()
        t = torch.empty(gain_offset + a.size, device="cuda")[gain_offset:].view(a.shape)
        t.copy_(on_gpu(torch, np.ascontiguousarray(a)))
        return t
    q_out = torch.full((b.n_tok, H, D), 7.0, dtype=k.dtype, device="cuda") if with_q else None
    rope = None if axes is None else binding.RopeAxes(*axes)
    pool.append_norm(layer, batch_on_gpu(gpu, b, pos), dx[:, :H] if with_q else None, dx[:, H:H + G], dx[:, H + G:], q_out, q_gain=gain_on_gpu("q") if with_q else None,
                     k_gain=gain_on_gpu("k"), eps=eps, positions=None if positions is None else on_gpu(torch, positions), axes=rope)
    pool.sync()
    where = np.concatenate([b.ctx[s] + np.arange(n) for s, n in enumerate(b.nodes)] + [np.zeros(b.n_tok - b.live, int)]) if pos is None else pos
    axis, rank = (np.zeros(D // 2, int), np.arange(D // 2)) if axes is None else (np.array(axes[0]), np.array(axes[1] if len(axes) > 1 else np.arange(D // 2)))
    table = np.stack([where] * 4) if positions is None else positions
    angle = np.where(axis >= 0, table[np.maximum(axis, 0)].T.astype(np.float64) * np.float64(np.float32(THETA)) ** (-2.0 * rank / D), 0.0)
    half = _paged.HALF_STEP[b.dtype]
    new_k, new_v = k.float().cpu().numpy(), v.float().cpu().numpy()
    want_k, want_v = b.k.copy(), b.v.copy()
    parts = {}
    for n, at in (("q", slice(0, H)), ("k", slice(H, H + G))):
        want, y = _prefix.norm_and_turn(x[:, at], gain[n], eps, angle, mode)
        # products and sums of the norm and of the rotation in 32 bits (below 2^-19 of both members of a pair), one rounding;
        # binary16 below its normal numbers 2^-25
        big = np.abs(y)
        partner = np.roll(big, D // 2, -1) if mode == 0 else big.reshape(*big.shape[:-1], D // 2, 2)[..., ::-1].reshape(big.shape)
        parts[n] = want, np.abs(want) * half + (big + partner) * 2.0 ** -19 + 2.0 ** -25
    for s, n in enumerate(b.nodes):
        for i in range(n):
            page, row = b.place(s, int(b.ctx[s]) + i)
            t = int(b.row_begin[s]) + i
            assert np.all(np.abs(new_k[layer, page, :, row] - parts["k"][0][t]) <= parts["k"][1][t])
            want_k[layer, page, :, row] = new_k[layer, page, :, row]
            want_v[layer, page, :, row] = _paged.rounded(x[t, H + G:], b.dtype)
    assert np.array_equal(new_k, want_k) and np.array_equal(new_v, want_v)      # nothing else has changed
    if with_q:
        got = q_out.float().cpu().numpy()
        assert np.all(np.abs(got[:b.live] - parts["q"][0][:b.live]) <= parts["q"][1][:b.live])
        assert np.all(got[b.live:] == 7.0)
        return got


def three(rs, n):
    return rs.randint(-50, 5000, (3, n)).astype(np.int32)


@pytest.mark.parametrize("dtype,src", [("float16", "float32"), ("float16", "float16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
@pytest.mark.parametrize("dim,mode,page", [(128, 0, 16), (64, 1, 8), (128, 1, 32), (64, 0, 16)])
@pytest.mark.parametrize("gains", ["shared", "each"])
def test_types_and_layouts(gpu, dtype, src, dim, mode, page, gains):
    b = Batch(500, ctx=[0, 30, 7], nodes=[3, 1, 6], page=page, layers=2, kv_heads=2, q_heads=6, dim=dim, dtype=dtype, pad=2)
    check(gpu, b, src, mode, gains, axes=([i % 3 for i in range(dim // 2)],), positions=three(b.rs, b.n_tok), layer=1)


@pytest.mark.parametrize("gains", ["q", "k", "none"])
def test_only_some_heads_are_normed(gpu, gains):
    b = Batch(501, ctx=[5, 0], nodes=[2, 9], page=8, kv_heads=3, q_heads=3, dim=64)
    check(gpu, b, "float32", 0, gains)


def test_without_gains_and_axes_it_is_the_plain_append(gpu):
    torch, binding = gpu
    b = Batch(502, ctx=[5, 300], nodes=[2, 9], page=16, kv_heads=2, q_heads=4, dim=128)
    x = torch.randn((b.n_tok, 8, 128), device="cuda")
    seen = []
    for call in ("append", "append_norm"):
        k, v, pool = cache_on_gpu(gpu, b, THETA)
        q = torch.empty((b.n_tok, 4, 128), dtype=torch.float16, device="cuda")
        getattr(pool, call)(0, batch_on_gpu(gpu, b), x[:, :4], x[:, 4:6], x[:, 6:], q)
        pool.sync()
        seen.append((q, k, v))
    assert all(torch.equal(a, c) for a, c in zip(*seen))


@pytest.mark.parametrize("axes", [([-1] * 32,), ([0] * 16 + [-1] * 16,), ([1] * 32, [2 * (i % 16) for i in range(32)]), ([3, 2, 1, 0] * 8, list(range(31, -1, -1)))])
def test_pairs_that_do_not_turn_and_frequencies_of_their_own(gpu, axes):
    b = Batch(503, ctx=[5], nodes=[7], page=8, kv_heads=1, q_heads=2, dim=64)
    check(gpu, b, "float32", 0, axes=axes, positions=b.rs.randint(0, 100000, (4, 7)).astype(np.int32))
    check(gpu, b, "float32", 1, axes=axes, pos=np.arange(100, 107).astype(np.int32))


@pytest.mark.parametrize("offset,gain_offset", [(0, 1), (1, 0), (3, 2), (8, 4)])
@pytest.mark.parametrize("src", ["float32", "float16"])
def test_unaligned_sources_and_gains(gpu, offset, gain_offset, src):
    b = Batch(504, ctx=[9, 1], nodes=[4, 3], page=16, kv_heads=2, q_heads=5 - 1, dim=128)
    check(gpu, b, src, 0, "each", offset=offset, gain_offset=gain_offset)


def test_many_rows_take_a_warp_each(gpu):
    """More rows than a CTA each pays for (16 for each of the 148 SMs)."""
    b = Batch(505, ctx=[0, 5], nodes=[2400, 3], page=32, kv_heads=1, q_heads=2, dim=64, dtype="bfloat16", pad=1)
    check(gpu, b, "bfloat16", 0, "shared", axes=([0] * 8 + [1] * 12 + [2] * 12,), positions=three(b.rs, b.n_tok))


def test_heads_of_zeros_and_of_large_and_small_numbers(gpu):
    b = Batch(506, ctx=[3], nodes=[5], page=8, kv_heads=2, q_heads=2, dim=64, dtype="bfloat16")
    x = b.rs.standard_normal((5, 6, 64)).astype(np.float32)
    x *= np.array([0.0, 1e-12, 1.0, 1e4, 1e12])[:, None, None].astype(np.float32)
    got = check(gpu, b, "float32", 0, "shared", x=x, eps=1e-6)
    assert np.all(got[0] == 0)


def test_no_queries_and_one_row(gpu):
    check(gpu, Batch(507, ctx=[31], nodes=[1], page=8, kv_heads=8, q_heads=8, dim=128), "float16", 0, with_q=False)
    check(gpu, Batch(508, ctx=[0], nodes=[1], page=8, kv_heads=1, q_heads=1, dim=64), "float32", 1)


def test_far_positions(gpu):
    """The fraction of a turn is formed in 64 bits: 2^28 positions away it is as good as near."""
    b = Batch(509, ctx=[3], nodes=[4], page=8, kv_heads=1, q_heads=1, dim=64)
    check(gpu, b, "float32", 0, "none", positions=np.array([[0, 1 << 20, (1 << 28) + 1, -(1 << 27)]], np.int32))


def test_bad_entries_are_skipped(gpu):
    torch, binding = gpu
    b = Batch(510, ctx=[3, 900, 2], nodes=[2, 1, 2], page=8, kv_heads=1, q_heads=2, dim=64)
    k, v, pool = cache_on_gpu(gpu, b, THETA)
    table = b.table.copy()
    table[0, 0] = 10 ** 6
    x = torch.randn((5, 4, 64), device="cuda")
    q, gain = torch.zeros((5, 2, 64), dtype=torch.float16, device="cuda"), torch.ones(64, device="cuda")
    batch = binding.PagedBatch(on_gpu(torch, table[:, :20]), on_gpu(torch, b.row_begin), on_gpu(torch, b.ctx), 5)
    pool.append_norm(0, batch, x[:, :2], x[:, 2:3], x[:, 3:], q, q_gain=gain, k_gain=gain)
    with pytest.raises(binding.PrimaError) as e:
        pool.sync()
    assert "page" in str(e.value) and "slot" in str(e.value)
    changed = (k.float().cpu().numpy() != b.k).any((0, 2, 3, 4))
    assert set(np.flatnonzero(changed)) <= {int(b.table[2, 0])} and (q[0] != 0).any()


def test_argument_errors(gpu):
    torch, binding = gpu
    b = Batch(511, ctx=[3], nodes=[2], page=8, kv_heads=1, q_heads=2, dim=64)
    k, v, pool = cache_on_gpu(gpu, b, THETA)
    batch = batch_on_gpu(gpu, b)
    x, q = torch.zeros((2, 4, 64), device="cuda"), torch.empty((2, 2, 64), dtype=torch.float16, device="cuda")
    gain = torch.ones(64, device="cuda")

    def call(**kw):
        pool.append_norm(0, batch, x[:, :2], x[:, 2:3], x[:, 3:], q, **{"q_gain": gain, **kw})
    call()
    for kw in (dict(q_gain=gain[:63]), dict(q_gain=gain.half()), dict(k_gain=torch.ones((2, 64), device="cuda")), dict(positions=torch.zeros((1, 3), dtype=torch.int32, device="cuda")),
               dict(positions=torch.zeros((1, 2), device="cuda")), dict(positions=torch.zeros((5, 2), dtype=torch.int32, device="cuda")),
               dict(axes=binding.RopeAxes([0] * 64)), dict(axes=binding.RopeAxes([1] * 32), positions=torch.zeros((1, 2), dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        with pytest.raises(binding.PrimaError) as e:
            call(**kw)
        assert e.value.code == binding.ERR_ARG
    for axis, rank in (([4] * 32, None), ([-2] * 32, None), ([0] * 31, None), ([0] * 32, [32] * 32)):
        with pytest.raises(ValueError):
            binding.RopeAxes(axis, rank)
    pool.sync()
