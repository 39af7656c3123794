"""Model steps over a paged cache, tree decoding and beam search on the GPU, against the CPU checker."""
import numpy as np
import pytest

import oracle
from paper_2504_08791_b200 import synth

pytestmark = pytest.mark.gpu

HIDDEN_TOL, LOGIT_TOL = 2e-3, 2e-2
MARGIN = 4e-2      # twice the logit tolerance: below this gap the two sides may legitimately choose differently


@pytest.fixture(scope="module")
def gpu():
    import torch
    from paper_2504_08791_b200 import binding
    assert torch.cuda.is_available()
    binding.lib()
    return torch, binding


def load(gpu, cfg, seed, checkers=()):
    torch, binding = gpu
    ctx = binding.Context(cfg)
    for layer, tid, rows, cols, data in synth.iter_model_tensors(seed, cfg):
        ctx.load(layer, tid, data, rows, cols)
        for c in checkers:
            c.load(layer, tid, data, rows, cols)
    return ctx


def stepper(gpu, ctx, n_pages=64, page=16, dtype=None, windows=None):
    torch, binding = gpu
    from paper_2504_08791_b200.paged import PagedStepper
    cfg = ctx.cfg
    shape = (cfg["n_layers"], n_pages, cfg["n_kv_heads"], page, cfg["head_dim"])
    k, v = (torch.full(shape, float("nan"), dtype=dtype or torch.float16, device="cuda") for _ in range(2))      # whatever is read was written before
    return PagedStepper(ctx, k, v, windows)


def rel(got, want):
    rms = np.sqrt(np.mean(want.astype(np.float64) ** 2, axis=-1, keepdims=True))
    return float((np.abs(got.astype(np.float64) - want) / rms).max())


@pytest.mark.parametrize("name,page,mode", [("tiny", 16, 0), ("small", 8, 0), ("tiny", 64, 1)])
def test_a_tree_step_matches_the_checker_along_every_branch(gpu, name, page, mode):
    """Prompt read through the paged path, then one step over a tree: every node's hidden state and logits are those of
    the checker run over the node's own branch; the accepted branch then continues like a plain sequence."""
    torch, binding = gpu
    from paper_2504_08791_b200.paged import DraftTree
    cfg = synth.model_config(name, max_n_tok=16, rope_mode=mode)
    L = cfg["n_layers"]
    check = oracle.Model(cfg)
    ctx = load(gpu, cfg, 41, [check])
    m = stepper(gpu, ctx, page=page, windows=[0, 1, L])
    rs = np.random.RandomState(2)
    prompt = [int(x) for x in rs.randint(0, cfg["vocab"], 21)]
    pages = []
    length = m.prefill(prompt, pages)
    check.forward_window(0, L, check.embed(prompt), 0)
    parents = [-1, 0, 0, 1, 1, 2, 3, 6, 0, 5, 9]
    tree = DraftTree([int(x) for x in rs.randint(0, cfg["vocab"], len(parents))], parents)
    n = len(parents)
    m.pages.grow(pages, length + n)
    batch = m.batch([pages], [length], [n], pos=[length + d for d in tree.depths()], mask=tree.mask())
    logits = m.step(tree.tokens, batch).cpu().numpy()
    hidden = m.hid[:n].cpu().numpy()
    m.pool.sync()
    ctx.sync()
    for i in range(n):
        path = [a for a in range(n) if int(tree.mask()[i, 0]) >> a & 1]
        want = check.forward_window(0, L, check.embed([tree.tokens[a] for a in path]), length)[-1:]      # overwrites the branch before
        assert rel(hidden[i:i + 1], want) <= HIDDEN_TOL
        assert np.abs(logits[i] - check.logits(want)[0]).max() <= LOGIT_TOL
    # the branch of node 7 is accepted; the next token goes behind it
    path = [0, 1, 3, 6, 7]
    m.pool.accept(batch, m._gpu([path]), m._gpu([len(path)]))
    check.forward_window(0, L, check.embed([tree.tokens[a] for a in path]), length)
    length += len(path)
    nxt = [int(x) for x in rs.randint(0, cfg["vocab"], 3)]
    m.pages.grow(pages, length + 3)
    got = m.step(nxt, m.batch([pages], [length], [3])).cpu().numpy()
    want = check.logits(check.forward_window(0, L, check.embed(nxt), length))
    m.pool.sync()
    assert np.abs(got - want).max() <= LOGIT_TOL
    check.close()
    ctx.close()


def test_ragged_batch_over_one_pool_and_padding(gpu):
    """Three sequences of different lengths in one step (two tokens, none, one), a padded row behind them."""
    torch, binding = gpu
    cfg = synth.model_config("tiny", max_n_tok=8)
    L = cfg["n_layers"]
    checks = [oracle.Model(cfg) for _ in range(3)]
    ctx = load(gpu, cfg, 43, checks)
    m = stepper(gpu, ctx, page=8, dtype=torch.float16)
    rs = np.random.RandomState(4)
    rows, lengths = [[], [], []], []
    for s, n in enumerate((5, 9, 16)):
        prompt = [int(x) for x in rs.randint(0, cfg["vocab"], n)]
        lengths.append(m.prefill(prompt, rows[s]))
        checks[s].forward_window(0, L, checks[s].embed(prompt), 0)
    counts, toks = [2, 0, 1], [int(x) for x in rs.randint(0, cfg["vocab"], 3)]
    for s in range(3):
        m.pages.grow(rows[s], lengths[s] + counts[s])
    batch = binding.PagedBatch(m.table_of(rows), m._gpu([0, 2, 2, 3]), m._gpu(lengths), 4)
    logits = m.step(toks + [7], batch).cpu().numpy()
    m.pool.sync()
    ctx.sync()
    for s, part in ((0, slice(0, 2)), (2, slice(2, 3))):
        want = checks[s].logits(checks[s].forward_window(0, L, checks[s].embed(toks[part]), lengths[s]))
        assert np.abs(logits[part] - want).max() <= LOGIT_TOL
    ctx.close()


@pytest.mark.parametrize("kind", ["alternatives", "wrong", "windows"])
def test_tree_decoding_gives_the_greedy_tokens(gpu, kind):
    torch, binding = gpu
    from paper_2504_08791_b200.paged import DraftTree, TreeSpeculativeDecoder
    cfg = synth.model_config("small", max_n_tok=16)
    L = cfg["n_layers"]
    check = oracle.Model(cfg)
    ctx = load(gpu, cfg, 19, [check])
    m = stepper(gpu, ctx, windows=[0, 2, L] if kind == "windows" else None)
    prompt = [int(x) for x in np.random.RandomState(6).randint(0, cfg["vocab"], 12)]
    h = check.forward_window(0, L, check.embed(prompt), 0)
    want, margins, pos = [], [], len(prompt)
    tok, margin = oracle.argmax(check.logits(h[-1:])[0])
    for _ in range(20):
        want.append(int(tok))
        margins.append(float(margin))
        tok, margin = oracle.argmax(check.logits(check.forward_window(0, L, check.embed([want[-1]]), pos))[0])
        pos += 1
    sure = next((i for i, x in enumerate(margins) if x <= MARGIN), 20)
    assert sure >= 6
    answers = {len(prompt) + i: t for i, t in enumerate(want)}
    rs = np.random.RandomState(8)

    def propose(history, limit):
        """Two alternatives at each of four depths; one of them is right, or none."""
        tokens, parents, line = [history[-1]], [-1], 0
        for d in range(4):
            right = answers.get(len(history) + d, 0)
            pair = [int(rs.randint(cfg["vocab"])), right] if kind != "wrong" else [(right + 1) % cfg["vocab"], (right + 2) % cfg["vocab"]]
            at = len(tokens)
            tokens += pair
            parents += [line, line]
            line = at + 1
        return DraftTree(tokens, parents)
    pages = []
    length = m.prefill(prompt[:-1], pages)
    out, stats = TreeSpeculativeDecoder(m, propose).generate(prompt, pages, length, 20)
    m.pool.sync()
    assert out[:sure] == want[:sure]
    if kind != "wrong":
        assert stats.cycles <= 20 - sure + (sure + 4) // 5
    check.close()
    ctx.close()


def test_beam_search_against_the_checker(gpu):
    """The beams' scores are the checker's scores of their tokens, and no continuation that the checker ranks clearly
    higher was left out at any step."""
    torch, binding = gpu
    from paper_2504_08791_b200.paged import BeamDecoder
    cfg = synth.model_config("tiny", max_n_tok=8)
    L, n, steps = cfg["n_layers"], 4, 6
    check = oracle.Model(cfg)
    ctx = load(gpu, cfg, 47, [check])
    m = stepper(gpu, ctx, page=8, n_pages=40)
    prompt = [int(x) for x in np.random.RandomState(9).randint(0, cfg["vocab"], 11)]
    got = BeamDecoder(m, n).generate(prompt, steps)
    m.pool.sync()
    assert len(m.pages.free) == 40                      # every page has come back

    def log_probs(tokens):
        x = check.logits(check.forward_window(0, L, check.embed(prompt + tokens), 0)[-1:])[0].astype(np.float64)
        x -= x.max()
        return x - np.log(np.exp(x).sum())
    beams = [(0.0, [])]
    for step in range(steps):
        cand = [(s + p, t + [w]) for s, t in beams for w, p in enumerate(log_probs(t))]
        cand.sort(key=lambda c: -c[0])
        beams = cand[:n]
    tol = steps * 2 * LOGIT_TOL
    assert [len(t) for _, t in got] == [steps] * n and len({tuple(t) for _, t in got}) == n
    for s, t in got:
        want = sum(log_probs(t[:i])[t[i]] for i in range(steps))
        assert abs(s - want) <= tol
    assert [s for s, _ in got] == sorted([s for s, _ in got], reverse=True)
    for (s, _), (want, _) in zip(got, beams):
        assert abs(s - want) <= tol                     # clearly better ones would show as higher scores
    # with an end token: a beam that ends keeps its score and takes no more tokens
    end = got[0][1][1]
    ended = BeamDecoder(m, n, end_token=end).generate(prompt, steps)
    assert any(t and t[-1] == end and len(t) < steps for _, t in ended)
    for s, t in ended:
        assert end not in t[:-1]
        assert abs(s - sum(log_probs(t[:i])[t[i]] for i in range(len(t)))) <= tol
    assert len(m.pages.free) == 40
    check.close()
    ctx.close()


def test_window_refusals_and_injected_failures(gpu):
    torch, binding = gpu
    cfg = synth.model_config("tiny", max_n_tok=4)
    ctx = load(gpu, cfg, 43)
    m = stepper(gpu, ctx, page=8)
    pages = []
    m.pages.grow(pages, 16)
    good = m.batch([pages], [0], [2])
    h = torch.zeros((4, cfg["hidden"]), device="cuda")
    shape = list(m.pool._keep[0].shape)

    def pool(theta=cfg["rope_theta"], **change):
        s = [change.get(n, x) for n, x in zip(("L", "pages", "G", "P", "D"), shape)]
        k, v = (torch.zeros(s, dtype=torch.float16, device="cuda") for _ in range(2))
        return binding.PagedCache(k, v, rope_theta=theta, rope_mode=cfg.get("rope_mode", 0))
    five = binding.PagedBatch(m.table_of([pages]), m._gpu([0, 5]), m._gpu([0]), 5)
    h5 = torch.zeros((5, cfg["hidden"]), device="cuda")
    for call in (lambda: ctx.forward_window_paged(m.pool, 0, cfg["n_layers"], h5, h5, five), lambda: ctx.forward_window_paged(m.pool, 1, 0, h, h, good),
                 lambda: ctx.forward_window_paged(m.pool, 0, cfg["n_layers"] + 1, h, h, good), lambda: ctx.forward_window_paged(pool(theta=7.0), 0, 1, h, h, good),
                 lambda: ctx.forward_window_paged(pool(D=64), 0, 1, h, h, good), lambda: ctx.forward_window_paged(pool(L=shape[0] - 1), 0, 1, h, h, good),
                 lambda: ctx.forward_window_paged(pool(G=shape[2] + 1), 0, 1, h, h, good)):
        with pytest.raises(binding.PrimaError) as e:
            call()
        assert e.value.code == binding.ERR_ARG
    for call in (lambda: ctx.forward_window_paged(m.pool, 0, 1, h[:1], h, good), lambda: ctx.forward_window_paged(m.pool, 0, 1, h[:, :256], h, good)):
        with pytest.raises(ValueError):
            call()
    # a launch refused in mid-window leaves the context usable, with the bits of a fresh one
    tok = [3, 5]
    want = m.step(tok, good).clone()
    for after in (1, 2, 3, 5, 9):
        ctx.embed(tok, m.hid[:2])
        ctx.set_option(binding.OPT_FAIL_AFTER_LAUNCHES, after)
        with pytest.raises(binding.PrimaError) as e:
            ctx.forward_window_paged(m.pool, 0, cfg["n_layers"], m.hid[:2], m.hid[:2], good)
        assert "injected" in str(e.value)
        ctx.set_option(binding.OPT_FAIL_AFTER_LAUNCHES, -1)
        assert torch.equal(m.step(tok, good), want)
    ctx.close()
