"""A step of drafted decoding written out on the host, in 64 bits: what rows of a tree see, and which drafts stay."""
import random

import torch


def parent_of(given, i):
    """what is no earlier row is none"""
    return given if 0 <= given < i else -1


def seen_rows(parents):
    """per row the rows that it sees: itself and its ancestors"""
    out = []
    for i, given in enumerate(parents):
        p = parent_of(given, i)
        out.append((out[p] if p >= 0 else frozenset()) | {i})
    return out


def words_of(rows, words):
    """a set of rows as signed words of 64 bits"""
    x = sum(1 << a for a in rows)
    parts = [(x >> (64 * w)) & ((1 << 64) - 1) for w in range(words)]
    return [p - (1 << 64) if p >> 63 else p for p in parts]


def distribution(scores, temperature):
    """softmax(scores / temperature) in 64 bits, all of it at the first maximum for temperature 0; None where there is none"""
    x = scores.double()
    if bool(torch.isnan(x).any()) or not bool(torch.isfinite(x.max())):
        return None
    if temperature == 0:
        p = torch.zeros_like(x)
        p[int((x == x.max()).nonzero()[0])] = 1.0
        return p
    e = torch.exp((x - x.max()) / temperature)
    return e / e.sum()


def draw(weights, v):
    """the first y whose running sum is above v of the whole"""
    upto = torch.cumsum(weights, 0)
    over = (upto > v * upto[-1]).nonzero()
    return int(over[0]) if len(over) else int((weights > 0).nonzero()[-1])


def walk(target, draft, tokens, parents, u, v, temperature, draft_temperature=1.0, distinct=False):
    """(path, next token) of one document; target and draft [rows, V], draft None where its tokens were picked"""
    n, V = target.shape
    path = [0]
    while True:
        node = path[-1]
        p = distribution(target[node], temperature)
        if p is None:
            return path, -1
        q = distribution(draft[node], draft_temperature) if draft is not None else None
        r, taken = p, -1
        for c in range(node + 1, n):
            if parent_of(parents[c], c) != node or taken >= 0 or (draft is not None and q is None):
                continue
            x = tokens[c]
            if not 0 <= x < V:
                continue
            one = torch.zeros(V, dtype=torch.float64)
            one[x] = 1.0
            qc = one if draft is None else q
            if not float(qc[x]) > 0:
                continue
            if float(u[c]) * float(qc[x]) < float(r[x]):
                taken = c
                continue
            r = torch.clamp(r - qc, min=0.0) if draft is not None else torch.where(one > 0, 0.0, r)
            r = r / r.sum() if float(r.sum()) > 0 else r * 0
            if draft is not None and distinct:
                q = q * (1 - one)
                q = q / q.sum() if float(q.sum()) > 0 else q
        if taken < 0:
            return path, draw(r if float(r.sum()) > 0 else p, float(v))
        path.append(taken)


def random_parents(rng, n, shape):
    """parents of n rows; "forest" has roots beside row 0 and values that name no earlier row"""
    if n == 0:
        return []
    if shape == "chain":
        return list(range(-1, n - 1))
    if shape == "star":
        return [-1] + [0] * (n - 1)
    if shape == "level":
        return [-1] + [rng.randint(max(0, (i - 1) // 3 - 1), (i - 1) // 3) for i in range(1, n)]
    out = [-1] + [i - 1 if rng.random() < 0.6 else rng.randint(0, i - 1) for i in range(1, n)]
    if shape == "forest":
        for i in range(n):
            if rng.random() < 0.15:
                out[i] = rng.choice([-1, -7, i, i + 1, 1 << 30, -(1 << 31)])
    return out
