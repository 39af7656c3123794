"""The operators of long prompts and bounded caches in a row, as a server uses them: requests behind one shared prompt enter
their tokens with normed heads, attend, add up what their entries receive, and drop the least of them."""
import numpy as np
import pytest

from tests import _paged, _prefix
from tests.test_gpu_paged import gpu, on_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

THETA = 1e4


@pytest.mark.parametrize("dim,dtype,group", [(64, "float16", 2), (128, "bfloat16", 4)])
def test_steps_of_a_batch_with_a_shared_prompt_and_evictions(gpu, dim, dtype, group):
    torch, binding = gpu
    rs = np.random.RandomState(40)
    G, layers, seqs, page, budget, slots, prompt = 2, 2, 3, 16, 24, 48, 83
    H = G * group
    tdt = getattr(torch, dtype)
    per = slots // page
    n_pages = seqs * per + -(-prompt // page) + 1
    k, v = (torch.zeros((layers, n_pages, G, page, dim), dtype=tdt, device="cuda") for _ in range(2))
    pool = binding.PagedCache(k, v, rope_theta=THETA)
    ids = rs.permutation(n_pages).astype(np.int32)
    own_table, prompt_table = on_gpu(torch, ids[:seqs * per].reshape(seqs, per)), on_gpu(torch, ids[None, seqs * per:])
    gains = {n: (1 + 0.2 * rs.standard_normal(dim)).astype(np.float32) for n in "qk"}
    dev_gain = {n: on_gpu(torch, g) for n, g in gains.items()}
    axes = binding.RopeAxes([0, 1] * (dim // 4))

    def i32(x):
        return on_gpu(torch, np.array(x, np.int32))

    def turned(x, which, pos):
        """Normed and turned in 64 bits; pos [2, n]."""
        angle = pos[[0, 1] * (dim // 4)].T.astype(np.float64) * np.float64(np.float32(THETA)) ** (-2.0 * np.arange(dim // 2) / dim)
        return _prefix.norm_and_turn(x, gains[which][None], 1e-6, angle, 0)[0]

    def enter(layer, batch, x, pos, q_out):
        d = on_gpu(torch, x)
        pool.append_norm(layer, batch, d[:, :H], d[:, H:H + G], d[:, H + G:], q_out, q_gain=dev_gain["q"], k_gain=dev_gain["k"], positions=on_gpu(torch, pos.astype(np.int32)), axes=axes)

    # the shared prompt, entered once
    begin = binding.PagedBatch(prompt_table, i32([0, prompt]), i32([0]), prompt)
    shared = []
    for layer in range(layers):
        x = rs.standard_normal((prompt, H + 2 * G, dim)).astype(np.float32)
        pos = np.stack([np.arange(prompt), np.arange(prompt) // 3])
        enter(layer, begin, x, pos, torch.empty((prompt, H, dim), dtype=tdt, device="cuda"))
        shared.append((turned(x[:, H:H + G], "k", pos), x[:, H + G:].astype(np.float64)))
    prefix = binding.PrefixBatch(prompt_table, i32([prompt]), i32([0, seqs]))

    weight = torch.zeros((layers, seqs, G, slots), device="cuda")
    born = torch.zeros((layers, seqs, G, slots), dtype=torch.int32, device="cuda")
    length, entered = i32([0] * seqs), np.zeros(seqs, int)
    host = [[[dict(k=[], v=[], w=[], born=[]) for _ in range(G)] for _ in range(seqs)] for _ in range(layers)]
    half = _paged.HALF_STEP[dtype]
    evictions = 0
    for step in range(9):
        counts = rs.randint(0 if step else 1, 8, seqs)
        n = int(counts.sum())
        if n == 0:
            continue
        first = np.concatenate([[0], np.cumsum(counts)])
        seq = np.repeat(np.arange(seqs), counts)
        at = np.concatenate([entered[s] + np.arange(c) for s, c in enumerate(counts)])
        pos = np.stack([prompt + at, prompt // 3 + at])
        held = length.cpu().numpy().copy()
        batch = binding.PagedBatch(own_table, i32(first), length, n, pos=i32(pos[0]))
        for layer in range(layers):
            x = rs.standard_normal((n, H + 2 * G, dim)).astype(np.float32)
            q, out = (torch.empty((n, H, dim), dtype=tdt, device="cuda") for _ in range(2))
            lse = torch.empty((n, H), device="cuda")
            enter(layer, batch, x, pos, q)
            pool.prefix_attention(layer, batch, prefix, q, out, lse=lse)
            pool.attention_weights(layer, batch, q, lse, weight[layer], weight_in=weight[layer], born=born[layer])
            # the same in 64 bits, from the entries that are there in 64 bits
            kk, vv, qq = turned(x[:, H:H + G], "k", pos), x[:, H + G:].astype(np.float64), turned(x[:, :H], "q", pos)
            for t in range(n):
                for g in range(G):
                    e = host[layer][seq[t]][g]
                    e["k"].append(kk[t, g])
                    e["v"].append(vv[t, g])
                    e["w"].append(0.0)
                    e["born"].append(int(pos[0, t]))
            got, z = out.float().cpu().numpy(), lse.cpu().numpy()
            for t in range(n):
                for h in range(H):
                    g = h // group
                    e = host[layer][seq[t]][g]
                    own = held[seq[t]] + t - first[seq[t]] + 1
                    keys, values = np.concatenate([shared[layer][0][:, g], np.array(e["k"][:own])]), np.concatenate([shared[layer][1][:, g], np.array(e["v"][:own])])
                    s = keys @ qq[t, h] / dim ** 0.5
                    p = np.exp(s - s.max())
                    total = p.sum()
                    p /= total
                    # queries and keys are rounded to half a step each (of norms of about sqrt(dim): a score off by 2 half |q| |k| /
                    # sqrt(dim) at most), values and probabilities too; a weight is off by the factor exp(2 x that)
                    off = 2 * half * np.linalg.norm(qq[t, h]) * np.linalg.norm(keys, axis=1).max() / dim ** 0.5 + 2.0 ** -18
                    assert np.all(np.abs(got[t, h] - p @ values) <= (np.expm1(2 * off) + 3 * half) * (p @ np.abs(values)) + half * np.abs(p @ values) + 2.0 ** -24)
                    assert abs(z[t, h] - (s.max() + np.log(total))) <= off + 2.0 ** -18
                    for j in range(own):
                        e["w"][j] += p[shared[layer][0].shape[0] + j]
        length = length + i32(counts)
        entered += counts
        pool.sync()
        w, b, m = weight.cpu().numpy(), born.cpu().numpy(), length.cpu().numpy()
        for layer in range(layers):
            for s in range(seqs):
                for g in range(G):
                    e = host[layer][s][g]
                    assert len(e["k"]) == m[s] and b[layer, s, g, :m[s]].tolist() == e["born"]
                    # sums of probabilities that are off by the factors above: norms of queries and keys are below 1.6 sqrt(dim)
                    # (gains of 1 +- 0.2), so a score by 2 half 1.6^2 sqrt(dim); the choice is made of the kernel's own sums
                    assert np.all(np.abs(w[layer, s, g, :m[s]] - np.array(e["w"])) <= np.expm1(4 * half * 2.56 * dim ** 0.5) * np.array(e["w"]) + 1e-6)
        if (m > budget).any():
            evictions += 1
            recent = prompt + entered - 4
            pool.evict(own_table, length, weight, born, i32([budget] * seqs), length, first=prompt + 1, recent_from=i32(recent))
            pool.sync()
            for layer in range(layers):
                for s in range(seqs):
                    for g in range(G):
                        e = host[layer][s][g]
                        source = _prefix.choose(w[layer, s, g], b[layer, s, g], int(m[s]), budget, prompt + 1, int(recent[s]))[1]
                        for name in e:
                            e[name] = [e[name][j] for j in source]
            assert length.tolist() == np.minimum(m, budget).tolist()
    assert evictions >= 2
