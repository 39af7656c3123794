"""Host side of the paged loops: page counts, trees of drafted tokens, the tree decoder with a toy model."""
import numpy as np
import pytest

from paper_2504_08791_b200.paged import DraftTree, PageTable, TreeSpeculativeDecoder


def test_pages_are_taken_shared_and_given_back():
    t = PageTable(6, 4)
    a = []
    t.grow(a, 9)
    assert a == [0, 1, 2] and t.users[:3] == [1, 1, 1]
    t.grow(a, 12)
    assert len(a) == 3
    b = [t.share(p) for p in a]
    for p in a:
        t.drop(p)
    assert sorted(t.free) == [3, 4, 5] and t.users[:3] == [1, 1, 1]
    for p in b:
        t.drop(p)
    assert sorted(t.free) == list(range(6))
    with pytest.raises(RuntimeError):
        t.grow([], 25)


@pytest.mark.parametrize("seed", range(8))
def test_reordering_keeps_every_page_counted(seed):
    rs = np.random.RandomState(seed)
    t = PageTable(64, 4)
    rows, lengths = [], []
    for _ in range(4):
        r = []
        n = int(rs.randint(0, 14))
        t.grow(r, n)
        rows.append(r)
        lengths.append(n)
    for _ in range(10):
        parents = [int(p) for p in rs.randint(0, len(rows), 4)]
        old = [list(r) for r in rows]
        fresh = [t.take() for _ in range(4)]
        rows = t.reorder(rows, lengths, parents, fresh)
        for r, p in enumerate(parents):
            used = -(-lengths[p] // 4)
            first = p not in parents[:r]
            want = old[p][:used] if first or lengths[p] % 4 == 0 else old[p][:used - 1] + [fresh[r]]
            assert rows[r] == want
        lengths = [lengths[p] for p in parents]
        # a partly filled page belongs to one row alone, and the counts are the number of rows that name a page
        for r in range(4):
            if lengths[r] % 4:
                assert sum(rows[r][-1] in x for x in rows) == 1
        count = [sum(p in r for r in rows) for p in range(64)]
        assert count == t.users and sorted(t.free) == [p for p in range(64) if count[p] == 0]
        for r in range(4):
            lengths[r] += int(rs.randint(0, 3))
            t.grow(rows[r], lengths[r])


def test_tree_masks_and_acceptance():
    tree = DraftTree([7, 1, 2, 1, 5, 6], [-1, 0, 0, 1, 3, 2])
    assert tree.depths() == [0, 1, 1, 2, 3, 2]
    bits = [[a for a in range(6) if int(tree.mask()[i, 0]) >> a & 1] for i in range(6)]
    assert bits == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [0, 2, 5]]
    assert tree.accept([1, 1, 0, 9, 0, 0]) == ([0, 1, 3], 9)
    assert tree.accept([3, 0, 0, 0, 0, 0]) == ([0], 3)
    assert tree.accept([2, 0, 6, 0, 0, 4]) == ([0, 2, 5], 4)
    wide = DraftTree(list(range(70)), [-1] + list(range(69)))
    assert wide.mask().shape == (70, 2) and int(wide.mask()[69, 1].view(np.uint64)) == 63
    for parents in ([0], [-1, -1], [-1, 1], [-1, 2, 0]):
        with pytest.raises(ValueError):
            DraftTree(list(range(len(parents))), parents).mask()


class Toy:
    """A target whose next token depends on the whole history; its cache is a list of slots, and a step fails when a row
    would see a slot that does not hold its own history."""

    def __init__(self, max_n_tok=16):
        self.max_n_tok, self.slots, self.ctx, self.pool = max_n_tok, [], self, self
        self.pages, self._stream = PageTable(1000, 4), None
        self.steps = 0

    @staticmethod
    def next_of(history):
        h = 17
        for i, x in enumerate(history):
            h = (h * 1000003 + (x + 1) * (i + 7)) % 2147483647
        return h % 11

    def batch(self, rows, lengths, counts, pos=None, mask=None):
        return dict(length=lengths[0], n=counts[0], pos=pos, mask=mask)

    def step(self, tokens, batch):
        self.steps += 1
        del self.slots[batch["length"]:]
        self.slots += list(tokens)
        self.choices = []
        for i in range(batch["n"]):
            seen = [a for a in range(batch["n"]) if int(batch["mask"][i, a // 64]) >> (a % 64) & 1]
            history = self.slots[:batch["length"]] + [tokens[a] for a in seen]
            assert batch["pos"][i] == len(history) - 1
            self.choices.append(self.next_of(history))

    def argmax(self, logits, n):
        return np.array(self.choices[:n])

    def _gpu(self, a):
        return a

    def accept(self, batch, path, path_len, stream=None):
        keep = [self.slots[batch["length"] + a] for a in path[0]]
        self.slots[batch["length"]:] = keep


@pytest.mark.parametrize("kind", ["right", "wrong", "mixed", "alone"])
def test_tree_decoding_gives_the_targets_own_tokens(kind):
    prompt = [3, 1, 4, 1, 5]
    want, h = [], list(prompt)
    for _ in range(40):
        want.append(Toy.next_of(h))
        h.append(want[-1])
    rs = np.random.RandomState(5)

    def propose(history, limit):
        tokens, parents = [history[-1]], [-1]
        if kind == "alone":
            return DraftTree(tokens, parents)
        lines = {0: list(history)}
        while len(tokens) < limit:
            p = int(rs.randint(len(tokens)))
            right = Toy.next_of(lines[p])
            tok = right if kind == "right" or (kind == "mixed" and rs.rand() < 0.5) else (right + 1 + int(rs.randint(10))) % 11
            if any(parents[i] == p and tokens[i] == tok for i in range(len(tokens))):
                break      # another word in its place might be the right one
            lines[len(tokens)] = lines[p] + [tok]
            tokens.append(tok)
            parents.append(p)
        return DraftTree(tokens, parents)
    toy = Toy()
    toy.slots = list(prompt[:-1])
    out, stats = TreeSpeculativeDecoder(toy, propose).generate(prompt, [], len(prompt) - 1, 40)
    assert out == want
    assert sum(stats.per_cycle) >= 40 and toy.steps == stats.cycles
    if kind in ("wrong", "alone"):
        assert stats.cycles == 40
    if kind == "right":
        assert stats.cycles < 25


def test_a_draft_that_does_not_fit_is_refused():
    toy = Toy(4)
    toy.slots = [1]
    for bad in (DraftTree([9], [-1]), DraftTree([2, 1, 1, 1, 1], [-1, 0, 1, 2, 3]), DraftTree([], [])):
        with pytest.raises(ValueError):
            TreeSpeculativeDecoder(toy, lambda h, n: bad).generate([1, 2], [], 1, 3)


def test_a_context_knows_the_stream_it_was_made_on(monkeypatch):
    """Selection and accepted paths have to follow its steps, whatever torch's current stream is by then."""
    import torch
    from paper_2504_08791_b200 import binding, synth

    class Stream:
        def __init__(self, raw):
            self.cuda_stream = raw

    class Lib:
        def prima_ctx_create(self, cfg, stream, out):
            self.got = stream.value
            return 0

        def prima_ctx_destroy(self, h):
            return 0
    fake = Lib()
    monkeypatch.setattr(binding, "lib", lambda: fake)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(1234))
    for given, raw in ((None, 1234), (Stream(99), 99)):
        ctx = binding.Context(synth.model_config("tiny"), stream=given)
        assert fake.got == raw and ctx._stream.cuda_stream == raw
