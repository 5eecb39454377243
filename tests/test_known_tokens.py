"""Known tokens in a step of drafted tokens (the rest of a prompt, a token that was sampled elsewhere): what makes the
acceptance keep them, by the definitions (no GPU), and what Server.verify refuses."""

import numpy as np
import pytest

import drafts_reference as D

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("seed", range(6))
def test_a_known_token_is_kept_when_the_choice_before_it_is_the_token_itself(seed):
    rng = np.random.default_rng(seed)
    add = rng.integers(1, 65, 20)
    known = np.array([rng.integers(1, n + 1) for n in add])
    first = np.concatenate([[0], np.cumsum(add)])
    parent = np.concatenate([D.tree(rng, n, 4) for n in add])
    token, choice = rng.integers(0, 2, (2, len(parent)))
    length = add + rng.integers(0, 50, 20)
    model = choice.copy()
    for r in range(20):
        for i in range(known[r] - 1):
            parent[first[r] + i + 1], choice[first[r] + i] = i, token[first[r] + i + 1]
    path, kept, after, left = D.accept(first, length, parent, token, choice)
    seen, position = D.plan(first, length, parent)
    for r in range(20):
        f, n = first[r], known[r]
        assert kept[r] >= n and path[f:f + n] == list(range(n)) and left[r] == length[r] - add[r] + kept[r]
        assert after[r] == model[f + path[f + kept[r] - 1]]                          # the model's own choice
        assert [position[f + i] - position[f] for i in range(n)] == list(range(n))
        assert [seen[f + i] for i in range(n)] == [2 ** (i + 1) - 1 for i in range(n)]


@pytest.mark.parametrize("add,known", [([3, 4], [3]), ([3, 4], [4, 0]), ([3, 4], [-1, 0]), ([70, 4], [69, 4]), ([70, 4], [0, 1]),
                                       ([3, 4], [[3, 4]])])
def test_counts_of_known_tokens_that_are_refused(monkeypatch, add, known):
    from paper_2606_30391_amd import festina
    from paper_2606_30391_amd.serve import Server
    srv = object.__new__(Server)
    srv.blocks = srv.drafts = None
    monkeypatch.setattr(Server, "_begin", lambda self, add: pytest.fail("the step has begun"))
    monkeypatch.setattr(festina, "_check", lambda *a: None)
    with pytest.raises(ValueError, match="known"):
        srv.verify(add, None, None, None, None, known=known)
