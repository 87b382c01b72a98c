"""The host's statement of drafted decoding: what it must be whatever computes it."""
import itertools
import math
import random

import pytest
import torch

import draft_reference as ref


@pytest.mark.parametrize("mode", ["drawn", "distinct", "picked"])
def test_the_next_token_has_the_targets_distribution(mode):
    """One level of a tree, two siblings over four tokens, every number's whole range: drafts by their probabilities, random numbers
    on a grid of N midpoints.  A token's share differs from the target's probability only by the grid: a threshold is off by at most
    half a cell, 1 / 2N, for each of the two accepting numbers, once more for how often the final one is asked, and its interval has
    two ends: 2.5 / N."""
    V, N, siblings = 4, 12, 2
    g = torch.Generator().manual_seed(4)
    target, draft = torch.randn(1 + siblings, V, generator=g), torch.randn(1 + siblings, V, generator=g)
    q = ref.distribution(draft[0], 1.0).tolist()
    p = ref.distribution(target[0], 0.8)
    grid = [(i + 0.5) / N for i in range(N)]
    share = torch.zeros(V, dtype=torch.float64)
    if mode == "picked":
        drafts = [((1, 3), 1.0)]
    else:
        drafts = []
        for x in itertools.product(range(V), repeat=siblings):
            if mode == "distinct" and len(set(x)) < siblings:
                continue
            w, left = 1.0, 1.0
            for t in x:
                w *= q[t] / left
                left -= q[t] if mode == "distinct" else 0.0
            drafts.append((x, w))
    assert abs(sum(w for _, w in drafts) - 1) < 1e-12
    for x, w in drafts:
        for u in itertools.product(grid, repeat=siblings):
            tokens = (0,) + x
            path, token = ref.walk(target, None if mode == "picked" else draft, tokens, [-1] + [0] * siblings, (0.5,) + u, 0.5, 0.8, 1.0, mode == "distinct")
            if len(path) > 1:
                share[tokens[path[1]]] += w / N ** siblings
            else:                                      # the final number's whole range at once
                for v in grid:
                    _, token = ref.walk(target, None if mode == "picked" else draft, tokens, [-1] + [0] * siblings, (0.5,) + u, v, 0.8, 1.0, mode == "distinct")
                    share[token] += w / N ** (siblings + 1)
    assert float((share - p).abs().max()) <= 2.5 / N, (share, p)


def test_rows_see_their_ancestors():
    assert ref.seen_rows([-1, 0, 1, 0, 3, -1, 6, 9]) == [{0}, {0, 1}, {0, 1, 2}, {0, 3}, {0, 3, 4}, {5}, {6}, {7}]
    assert ref.words_of({0, 63, 64}, 2) == [-(1 << 63) + 1, 1]
    rng = random.Random(1)
    for shape in ("chain", "star", "level", "deep", "forest"):
        parents = ref.random_parents(rng, 70, shape)
        for i, rows in enumerate(ref.seen_rows(parents)):
            a, up = i, set()
            while a >= 0:
                up.add(a)
                a = ref.parent_of(parents[a], a)
            assert rows == up


def test_borders():
    t = torch.tensor([[0.0, 0.0, -math.inf], [0.0, 0.0, 0.0]])
    assert ref.walk(t, None, (0, 2), [-1, 0], (0, 0), 0.0, 1.0) == ([0], 0)          # no probability: refused whatever the number
    assert ref.walk(t, None, (0, 1), [-1, 0], (0, 0.49), 0.4, 1.0) == ([0, 1], 1)
    assert ref.walk(t, None, (0, 1), [-1, 0], (0, 0.5), 0.99, 1.0) == ([0], 0)       # 1/2 < 1/2 is not
    assert ref.walk(t, None, (0, 1), [-1, 0], (0, 0.0), 0.0, 0.0) == ([0], 0)        # the first of equals
    assert ref.walk(torch.tensor([[math.nan, 0.0]]), None, (0,), [-1], (0,), 0.0, 1.0) == ([0], -1)
