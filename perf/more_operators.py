"""A step of drafted decoding over a paged cache, as cases that can be timed: what rows of a tree of drafted tokens see, their
attention over the cache, which of the drafts stay, and moving what stays to its place.

`own` false: the operators in elementary torch operations, in 32 bits (verification, where a token hangs on a border, in 64),
rounded once at the end.  `own` true: the calls that a program makes of `paper_2403_10616_amd`.  Sizes are those of the
library's own configurations, or generic ones around them.

A document's new rows are a tree: row 0 is the last token that is certain, every other row a drafted token whose parent is an
earlier row.

  tree    depth of every row, and as bits which rows of its document it sees: itself and its ancestors
  attend  attention of the rows over the cache: row i, at position cached + depth, sees cached position j where
          j > position - window or j < sinks, and the drafted rows of its bits
  verify  walks from row 0: a child is taken by the ratio of the target's probability to the draft's against a given random
          number; where none is taken the next token is drawn from what the target has left
  keep    the cache rows of the path that stays move behind the cached positions, in all layers
"""
import math
import random

import torch

own = False

DEV = "cuda"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_ANY = 1 << 30                    # a window that reaches everything


def _tree(name, batch, rows, shape, ragged):
    return dict(name=name, kind="tree", batch=batch, rows=rows, shape=shape, ragged=ragged)


def _attend(name, dtype, batch, rows, shape, cached, heads, kv_heads, d_head, page, window, sinks, ragged):
    return dict(name=name, kind="attend", dtype=dtype, batch=batch, rows=rows, shape=shape, cached=cached, heads=heads,
                kv_heads=kv_heads, d_head=d_head, page=page, window=window, sinks=sinks, ragged=ragged)


def _verify(name, dtype, batch, rows, shape, vocab, drafts, temperature, ragged):
    """drafts: how the drafted tokens came about: "drawn" (each from the draft's distribution), "distinct" (siblings drawn
    without replacement), "top" (the draft's most probable ones; its logits are not kept)"""
    return dict(name=name, kind="verify", dtype=dtype, batch=batch, rows=rows, shape=shape, vocab=vocab, drafts=drafts,
                temperature=temperature, ragged=ragged)


def _keep(name, dtype, batch, rows, cached, layers, kv_heads, d_head, page, ragged):
    return dict(name=name, kind="keep", dtype=dtype, batch=batch, rows=rows, cached=cached, layers=layers, kv_heads=kv_heads,
                d_head=d_head, page=page, ragged=ragged)


def listed():
    return [
        # One document is being continued with a small tree.  Latency.
        _tree("tree one document", 1, 16, "level", False),
        # Evaluation of many documents with large trees of every shape.
        _tree("trees large batch", 256, 500, "mixed", True),
        # A block of the 150M path, one document of 1000 positions, 16 drafted rows.  Latency.
        _attend("attention one document", "bf16", 1, 16, "level", 1000, 14, 14, 64, 16, _ANY, 0, False),
        # A serving batch with shared heads, trees of up to 64 rows over caches of every length.
        _attend("attention serving batch", "bf16", 32, 64, "mixed", 16000, 16, 4, 128, 64, _ANY, 0, True),
        # Two documents of the 150M path with large trees, under the window that it was trained with.
        _attend("attention large trees window", "bf16", 2, 400, "level", 12000, 14, 14, 64, 16, 2048, 4, False),
        # A small path in fp32: evaluation with drafts from a cheaper path.
        _attend("attention fp32", "f32", 5, 25, "mixed", 700, 8, 2, 32, 32, _ANY, 0, True),
        # One document, a chain of five drafts from a cheaper path.  Latency.
        _verify("verify one chain", "bf16", 1, 6, "chain", 32000, "drawn", 1.0, False),
        # A serving batch of chains.
        _verify("verify chains", "f32", 64, 8, "chain", 32000, "drawn", 0.9, True),
        # Trees of the draft's most probable tokens.
        _verify("verify trees of likely tokens", "bf16", 32, 64, "level", 32000, "top", 0.8, False),
        # Trees whose siblings were drawn without replacement, a vocabulary of odd size.
        _verify("verify distinct siblings", "f32", 24, 40, "level", 20011, "distinct", 1.0, True),
        # One document of the 150M path, all twelve blocks.  Latency.
        _keep("keep one document", "bf16", 1, 16, 1000, 12, 14, 64, 16, False),
        # A batch whose drafts went well, wide heads in 24 layers.
        _keep("keep batch", "bf16", 64, 60, 60, 24, 8, 128, 64, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_FLOPS, _MOST_BYTES, _MOST_STATE = 7.0e10, 4.5e8, 7.0e8      # the largest listed cases


def draw(rng):
    while True:
        kind = rng.choice(("tree", "attend", "attend", "verify", "verify", "keep"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        ragged, shape = rng.random() < 0.6, rng.choice(("chain", "level", "deep", "mixed"))
        if kind == "tree":
            case = _tree(None, _log_int(rng, 1, 256), _log_int(rng, 2, 500), rng.choice(("level", "deep", "mixed")), ragged)
        elif kind == "attend":
            kv = _log_int(rng, 1, 16)
            heads = kv * rng.choice((1, 1, 2, 3, 4, 8))
            rows = _log_int(rng, 1, 500)
            window = rng.choice((_ANY, max(rows, _log_int(rng, 16, 4096))))
            case = _attend(None, dtype, _log_int(rng, 1, 64), rows, shape, rng.choice((0, _log_int(rng, 1, 20000), _log_int(rng, 1, 20000))),
                           heads, kv, rng.choice((32, 64, 64, 128)), rng.choice((16, 32, 64, 128)), window,
                           rng.choice((0, _log_int(rng, 1, 128))), ragged)
            if heads > 32:
                continue
        elif kind == "verify":
            case = _verify(None, dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 64), shape, _log_int(rng, 100, 60000),
                           rng.choice(("drawn", "distinct", "top")), rng.choice((0.0, 0.6, 0.8, 1.0, 1.0, 1.3)), ragged)
        else:
            case = _keep(None, dtype, _log_int(rng, 1, 128), _log_int(rng, 1, 128), rng.choice((0, _log_int(rng, 1, 1000))),
                         _log_int(rng, 1, 24), _log_int(rng, 1, 16), rng.choice((32, 64, 128)), rng.choice((16, 32, 64, 128)), ragged)
        del case["name"]
        w = work(case)
        # the fp32 matrix cores are a sixteenth as fast as the bf16 ones
        if w["flops"] * (16 if case.get("dtype") == "f32" else 1) <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES and _state_bytes(case) <= _MOST_STATE:
            return case


# ---- what a case has whatever the seed of its data: lengths, trees, paths ---------------------------------------------
def _parents(rng, n, shape):
    """parents of rows 0 .. n - 1, the root's -1; no row has more than eight children"""
    if shape == "mixed":
        shape = rng.choice(("chain", "level", "deep"))
    if shape == "chain":
        return list(range(-1, n - 1))
    out, children, b = [-1] * min(n, 1), [0] * n, rng.randint(2, 4)
    for i in range(1, n):
        p = rng.randint(max(0, (i - 1) // b - 1), (i - 1) // b) if shape == "level" else i - 1 if rng.random() < 0.75 else rng.randint(0, i - 1)
        while children[p] == 8:
            p += 1
        children[p] += 1
        out.append(p)
    return out


def _depths(parents):
    out = []
    for p in parents:
        out.append(0 if p < 0 else out[p] + 1)
    return out


def _plan(case):
    """(cached positions, parents of the new rows) of every document; keep: (cached, path of rows that stay)"""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    docs = []
    for b in range(case["batch"]):
        first = b == 0 or not case["ragged"]
        n = case["rows"] if first else rng.randint(0, case["rows"])
        cached = case.get("cached", 0)
        cached = cached if first else rng.randint(0, cached)
        if case["kind"] != "keep":
            docs.append((cached, _parents(rng, n, case["shape"])))
            continue
        # Row 0 and some drafts stay.  The rows in front of the first gap keep their places; those behind it come from
        # behind all places, so that a pass repeated on its own result changes nothing.
        kept = min(n, rng.randint((n + 7) // 8, max(1, n // 2))) if n else 0
        still = rng.randint(1, kept) if kept and 2 * kept <= n else kept
        docs.append((cached, list(range(still)) + sorted(rng.sample(range(kept, n), kept - still))))
    return docs


def _starts(docs):
    out = [0]
    for _, rows in docs:
        out.append(out[-1] + len(rows))
    return out


def _words(case):
    return -(-case["rows"] // 64)


def _levels(case, docs):
    """rows that a walk visits, about: half the levels of each tree, and the one it ends at"""
    return sum(1 + max(_depths(p)) // 2 for _, p in docs if p)


def _element(case):
    return 4 if case["dtype"] == "f32" else 2


def _state_bytes(case):
    docs = _plan(case)
    if case["kind"] == "tree":
        return _starts(docs)[-1] * 8 * _words(case)
    if case["kind"] == "verify":
        return _starts(docs)[-1] * case["vocab"] * _element(case) * (1 if case["drafts"] == "top" else 2)
    ps, layers = case["page"], case.get("layers", 1)
    held = sum(-(-(c + (len(r) if case["kind"] == "attend" else case["rows"])) // ps) for c, r in docs) * ps
    return held * layers * 2 * case["kv_heads"] * case["d_head"] * _element(case)


def work(case):
    docs = _plan(case)
    rows = _starts(docs)[-1]
    if case["kind"] == "tree":
        return dict(bytes=rows * (8 + 8 * _words(case)), flops=0.0)
    es = _element(case)
    if case["kind"] == "verify":
        read = _levels(case, docs) * case["vocab"] * es * (1 if case["drafts"] == "top" else 2)
        return dict(bytes=read + rows * 12 + case["batch"] * (12 + 4 * case["rows"]), flops=0.0)
    Hkv, dh = case["kv_heads"], case["d_head"]
    if case["kind"] == "keep":
        moved = sum(i != r for _, path in docs for i, r in enumerate(path))
        return dict(bytes=max(1, moved) * case["layers"] * 4 * Hkv * dh * es, flops=0.0)
    H, W, K = case["heads"], case["window"], case["sinks"]
    seen = pairs = 0
    for c, parents in docs:
        if parents:
            first = max(0, c - W + 1)
            seen += c - first + min(K, first) + len(parents)
            for d in _depths(parents):
                near = min(c, max(0, c + d - W + 1))
                pairs += c - near + min(K, near) + d + 1
    return dict(bytes=seen * 2 * Hkv * dh * es + rows * (H * (2 * dh * es + 4) + 4 + 8 * _words(case)), flops=4.0 * dh * H * pairs)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(shape, device=DEV, generator=g)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _bits(parents, words):
    """which rows each row sees, as words of 64 bits (signed)"""
    seen, out = [], []
    for i, p in enumerate(parents):
        seen.append((1 << i) | (seen[p] if p >= 0 else 0))
        for w in range(words):
            x = (seen[i] >> (64 * w)) & ((1 << 64) - 1)
            out.append(x - (1 << 64) if x >> 63 else x)
    return out


def _table(g, case, used):
    """a table of pages in random order, a few pages more than are used"""
    per_doc, n_pages = max(max(used), 1) + 1, sum(used) + 3
    order = torch.randperm(n_pages, device=DEV, generator=g).tolist()
    table = torch.full((len(used), per_doc), -1, dtype=torch.int32)
    for b, n in enumerate(used):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    return table.to(DEV), n_pages, per_doc


def _cache(g, case, n_pages):
    """keys with a common part, values smaller: what a projection of normalised rows leaves"""
    Hkv, dh, ps = case["kv_heads"], case["d_head"], case["page"]
    cache = _randn(g, n_pages, 2, Hkv, ps, dh)
    cache[:, 0] += 0.5 * _randn(g, 1, Hkv, 1, dh)
    cache[:, 1] *= 0.5
    return cache.to(_TYPES[case["dtype"]])


def _drafted(g, s, draft, temperature):
    """the tokens that a draft with these logits proposes, row by row"""
    case, starts, docs = s["case"], s["starts"], s["docs"]
    tokens = torch.randint(0, case["vocab"], (starts[-1],), device=DEV, generator=g)
    child, parent, rank = [], [], []
    for b, (_, parents) in enumerate(docs):
        count = [0] * len(parents)
        for i, p in enumerate(parents):
            if p >= 0:
                child.append(starts[b] + i)
                parent.append(starts[b] + p)
                rank.append(count[p])
                count[p] += 1
    for lo in range(0, len(child), 256):
        at, up, nth = (torch.tensor(x[lo:lo + 256], device=DEV) for x in (child, parent, rank))
        scores = draft[up].float() / temperature
        if case["drafts"] == "drawn":                  # a Gumbel variable on each score: its largest is a draw
            scores -= torch.log(-torch.log(torch.rand(scores.shape, device=DEV, generator=g).clamp_(1e-30, 1 - 1e-7)))
            tokens[at] = scores.argmax(1)
        else:
            if case["drafts"] == "distinct":           # the same variables for all siblings: the next largest are draws without replacement
                first, which = torch.unique(up, return_inverse=True)
                noise = torch.stack([torch.rand(case["vocab"], device=DEV, generator=torch.Generator(device=DEV).manual_seed(s["seed"] * 4099 + int(r)))
                                     for r in first.tolist()])
                scores -= torch.log(-torch.log(noise.clamp_(1e-30, 1 - 1e-7)))[which]
            tokens[at] = torch.topk(scores, 8, 1).indices.gather(1, nth[:, None])[:, 0]
    return tokens.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    docs = _plan(case)
    s = dict(case=case, docs=docs, seed=int(seed), starts=_starts(docs))
    T, B, kind = s["starts"][-1], len(docs), case["kind"]
    s["row_start"] = _int32(s["starts"])
    s["cache_len"] = _int32([c for c, _ in docs])
    if kind == "verify":
        s["parent"] = _int32([p for _, parents in docs for p in parents])
    if kind == "tree":
        # other trees of the same sizes for other seeds
        rng = random.Random(int(seed))
        s["docs"] = docs = [(c, _parents(rng, len(parents), case["shape"])) for c, parents in docs]
        s["parent"] = _int32([p for _, parents in docs for p in parents])
        s["depth"] = torch.empty(T, dtype=torch.int32, device=DEV)
        s["seen"] = torch.empty((T, _words(case)), dtype=torch.int64, device=DEV)
        return s
    t = _TYPES[case["dtype"]]
    if kind == "verify":
        temperature = case["temperature"] or 1.0
        # scores of a model: a few tokens far above the rest; the target's are near the draft's
        draft = 3.0 * _randn(g, T, case["vocab"])
        target = (draft + 0.7 * _randn(g, T, case["vocab"])).to(t)
        draft = draft.to(t)
        s["tokens"] = _drafted(g, s, draft, temperature)
        s["target"], s["draft"] = target, None if case["drafts"] == "top" else draft
        s["u"], s["v"] = torch.rand(T, device=DEV, generator=g), torch.rand(B, device=DEV, generator=g)
        s["path"] = torch.empty((B, case["rows"]), dtype=torch.int32, device=DEV)
        s["kept"], s["next"] = (torch.empty(B, dtype=torch.int32, device=DEV) for _ in range(2))
        if own:
            import paper_2403_10616_amd as dp
            s["ws"] = torch.empty(dp.dipaco_k_draft_verify_workspace_bytes(T, B, case["vocab"]), dtype=torch.uint8, device=DEV)
        return s
    ps = case["page"]
    if kind == "keep":
        s["pages"], s["n_pages"], s["per_doc"] = _table(g, case, [-(-(c + case["rows"]) // ps) for c, _ in docs])
        s["caches"] = [_cache(g, case, s["n_pages"]) for _ in range(case["layers"])]
        s["path"] = _int32([path + [-1] * (case["rows"] - len(path)) for _, path in docs])
        s["kept"] = _int32([len(path) for _, path in docs])
        return s
    H, Hkv, dh = case["heads"], case["kv_heads"], case["d_head"]
    s["pages"], s["n_pages"], s["per_doc"] = _table(g, case, [-(-(c + len(p)) // ps) for c, p in docs])
    s["cache"] = _cache(g, case, s["n_pages"])          # the drafted rows' keys and values among them
    qkv = _randn(g, T, (H + 2 * Hkv) * dh)
    qkv[:, :H * dh] *= 1.5
    s["qkv"] = qkv.to(t)
    s["depth"] = _int32([d for _, parents in docs for d in _depths(parents)])
    s["seen"] = torch.tensor([x for _, parents in docs for x in _bits(parents, _words(case))], dtype=torch.int64).reshape(T, -1).to(DEV)
    s["o"], s["lse"] = torch.empty((T, H * dh), dtype=t, device=DEV), torch.empty((T, H), device=DEV)
    if own:
        import paper_2403_10616_amd as dp
        n = dp.dipaco_k_attention_tree_workspace_bytes(T, B, case["rows"], H, Hkv, dh, ps, s["per_doc"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------
def _padded(s):
    """[documents, rows] of a ragged batch: the row's index in the call (its last row behind the document's end), and whether there is one"""
    T, n = s["starts"][-1], s["case"]["rows"]
    first, count = s["row_start"][:-1, None].long(), (s["row_start"][1:] - s["row_start"][:-1])[:, None]
    i = torch.arange(n, device=DEV)[None, :]
    return (first + i).clamp(max=T - 1), i < count


def _plain_tree(s):
    n, (at, there) = s["case"]["rows"], _padded(s)
    i = torch.arange(n, device=DEV)
    jump = torch.where(there, s["parent"][at].long(), -1)
    jump = torch.where((jump >= 0) & (jump < i), jump, -1)
    sees = (i[:, None] == i[None, :]).expand(len(jump), n, n)
    for _ in range(max(1, n - 1).bit_length()):         # each round sees twice as far up
        far = jump.clamp(min=0)
        sees = sees | (sees.gather(1, far[:, :, None].expand(-1, -1, n)) & (jump >= 0)[:, :, None])
        jump = torch.where(jump >= 0, jump.gather(1, far), -1)
    words = _words(s["case"])
    wide = torch.zeros((*sees.shape[:2], 64 * words), dtype=torch.bool, device=DEV)
    wide[:, :, :n] = sees
    one = torch.ones((), dtype=torch.int64, device=DEV) << torch.arange(64, device=DEV)
    bits = (wide.reshape(*sees.shape[:2], words, 64) * one).sum(3)
    return (sees.sum(2) - 1).to(torch.int32)[there], bits[there]


def _plain_attend(s):
    case = s["case"]
    H, Hkv, dh, ps, W, K = case["heads"], case["kv_heads"], case["d_head"], case["page"], case["window"], case["sinks"]
    G = H // Hkv
    o = torch.zeros((s["starts"][-1], H * dh), dtype=s["qkv"].dtype, device=DEV)
    lse = torch.zeros((s["starts"][-1], H), device=DEV)
    for b, (c, parents) in enumerate(s["docs"]):
        n = len(parents)
        if not n:
            continue
        at = slice(s["starts"][b], s["starts"][b + 1])
        p, i = torch.arange(c + n, device=DEV), torch.arange(n, device=DEV)
        pos = (c + s["depth"][at].long())[:, None]
        drafted = (s["seen"][at][:, i // 64] >> (i % 64)) & 1 == 1
        sees = torch.cat([(p[None, :c] > pos - W) | (p[None, :c] < K), drafted], 1)
        kv = s["cache"][s["pages"][b][p // ps].long(), :, :, p % ps].float()          # [positions, 2, Hkv, dh]
        k, v = (kv[:, x].transpose(0, 1).contiguous() for x in (0, 1))
        q = s["qkv"][at, :H * dh].float().reshape(n, H, dh).transpose(0, 1).reshape(Hkv, G * n, dh)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()).reshape(H, n, c + n) / math.sqrt(dh)
        x = x.masked_fill_(~sees, -math.inf)
        top = x.amax(2, keepdim=True)
        e = torch.exp(x - top)
        total = e.sum(2, keepdim=True)
        ob = torch.matmul(e.reshape(Hkv, G * n, c + n), v).reshape(H, n, dh) / total
        o[at], lse[at] = ob.transpose(0, 1).reshape(n, -1).to(o.dtype), (top + torch.log(total))[:, :, 0].T
    return o, lse


def _distribution(logits, temperature):
    """[documents, vocabulary] in 64 bits; all of it at the first maximum where the temperature is 0"""
    x = logits.double()
    if temperature == 0:
        return torch.zeros_like(x).scatter_(1, x.argmax(1, keepdim=True), 1.0)
    e = torch.exp((x - x.amax(1, keepdim=True)) / temperature)
    return e / e.sum(1, keepdim=True)


def _plain_verify(s):
    case, T, B, n = s["case"], s["starts"][-1], len(s["docs"]), s["case"]["rows"]
    draft_temperature = case["temperature"] or 1.0
    at, there = _padded(s)
    # children[b, i, k]: the k-th child of row i of document b, or -1
    i = torch.arange(n, device=DEV)
    is_child = there[:, None, :] & (s["parent"][at][:, None, :] == i[None, :, None])      # [documents, row, child]
    order = is_child.cumsum(2) * is_child
    children = torch.full((B, n, 9), -1, device=DEV).scatter_(2, order, i.expand(B, n, n))[:, :, 1:]
    b = torch.arange(B, device=DEV)
    node, alive = torch.zeros(B, dtype=torch.long, device=DEV), there[:, 0]
    path, kept = torch.full((B, n), -1, device=DEV), alive.long()
    path[:, 0] = torch.where(alive, 0, -1)
    token = torch.full((B,), -1, device=DEV)
    for level in range(max(max(_depths(p), default=0) for _, p in s["docs"]) + 1):
        row = at[b, node]
        p = _distribution(s["target"][row], case["temperature"])
        q = None if s["draft"] is None else _distribution(s["draft"][row], draft_temperature)
        r, taken = p, torch.full((B,), -1, device=DEV)
        for k in range(8):
            child = children[b, node, k]
            up = at[b, child.clamp(min=0)]
            x = s["tokens"][up].long()[:, None]
            if q is None:
                qx = torch.ones_like(x, dtype=torch.float64)
                rest = r.scatter(1, x, 0.0)
            else:
                qx = q.gather(1, x)
                rest = (r - q).clamp_(min=0.0)
            tried = alive & (child >= 0) & (taken < 0) & (qx[:, 0] > 0)
            good = tried & (s["u"][up].double() * qx[:, 0] < r.gather(1, x)[:, 0])
            taken = torch.where(good, child, taken)
            total = rest.sum(1, keepdim=True)
            bad = (tried & ~good)[:, None]
            r = torch.where(bad, torch.where(total > 0, rest / total, 0.0), r)
            if case["drafts"] == "distinct":
                left = q.scatter(1, x, 0.0)
                total = left.sum(1, keepdim=True)
                q = torch.where(bad, torch.where(total > 0, left / total, 0.0), q)
        r = torch.where(r.sum(1, keepdim=True) > 0, r, p)
        upto = r.cumsum(1)
        above = upto > s["v"].double()[:, None] * upto[:, -1:]
        drawn = torch.where(above.any(1), above.to(torch.int8).argmax(1), case["vocab"] - 1)
        token = torch.where(alive & (taken < 0), drawn, token)
        alive = alive & (taken >= 0)
        if level + 1 < n:
            path[:, level + 1] = torch.where(alive, taken, -1)
        kept += alive
        node = torch.where(alive, taken, node)
    return path.to(torch.int32), kept.to(torch.int32), token.to(torch.int32)


def _plain_keep(s):
    case = s["case"]
    i = torch.arange(case["rows"], device=DEV)[None, :]
    ps, moves = case["page"], i < s["kept"][:, None]
    b = torch.arange(len(s["docs"]), device=DEV)[:, None].expand(moves.shape)[moves]
    to, frm = ((s["cache_len"][:, None] + x)[moves] for x in (i, s["path"]))
    to_page, from_page = (s["pages"][b, (x // ps).long()].long() for x in (to, frm))
    for cache in s["caches"]:
        cache[to_page, :, :, (to % ps).long()] = cache[from_page, :, :, (frm % ps).long()]
    return s["caches"]


_PLAIN = dict(tree=_plain_tree, attend=_plain_attend, verify=_plain_verify, keep=_plain_keep)


# ---- the calls a program makes --------------------------------------------------------------------------------------
def _own(s):
    import paper_2403_10616_amd as dp
    case, kind, T, B = s["case"], s["case"]["kind"], s["starts"][-1], len(s["docs"])
    n = case["rows"]
    if kind == "tree":
        dp.dipaco_k_draft_tree(s["parent"], s["row_start"], s["depth"], s["seen"], T, B, n)
        return s["depth"], s["seen"]
    dtype = dp.F32 if case["dtype"] == "f32" else dp.BF16
    if kind == "verify":
        dp.dipaco_k_draft_verify(dtype, s["target"], s["draft"], s["tokens"], s["parent"], s["row_start"], s["u"], s["v"], s["path"],
                                 s["kept"], s["next"], T, B, n, case["vocab"], case["temperature"], case["temperature"] or 1.0,
                                 case["drafts"] == "distinct", s["ws"])
        return s["path"], s["kept"], s["next"]
    Hkv, dh, ps = case["kv_heads"], case["d_head"], case["page"]
    if kind == "keep":
        dp.dipaco_k_cache_keep(dtype, s["path"], s["kept"], s["cache_len"], s["pages"], s["caches"], B, n, Hkv, dh, s["n_pages"], ps,
                               s["per_doc"])
        return s["caches"]
    dp.dipaco_k_attention_tree(dtype, s["qkv"], s["row_start"], s["cache_len"], s["depth"], s["seen"], s["pages"], s["cache"], s["o"],
                               s["lse"], T, B, n, case["heads"], Hkv, dh, s["n_pages"], ps, s["per_doc"], case["window"],
                               case["sinks"], s["ws"])
    return s["o"], s["lse"]


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ---- the definition, document by document -----------------------------------------------------------------------------
def _walk(s, b, rows, target, draft, u, tokens, parent):
    """(path, next token) of document b; rows: its rows' indices in the call"""
    case, temperature, path = s["case"], s["case"]["temperature"], [0]

    def softmax(x, t):
        x = x.double()
        if t == 0:
            p = torch.zeros_like(x)
            p[int((x == x.max()).nonzero()[0, 0])] = 1.0
            return p
        return torch.softmax(x / t, 0)

    while True:
        node = path[-1]
        p = softmax(target[rows[node]], temperature)
        q = softmax(draft[rows[node]], temperature or 1.0) if draft is not None else None
        left, taken = p.clone(), None
        for child in range(node + 1, len(rows)):
            if parent[rows[child]] != node:
                continue
            x = tokens[rows[child]]
            qx = 1.0 if q is None else float(q[x])
            if qx == 0.0:
                continue
            if u[rows[child]] * qx < float(left[x]):
                taken = child
                break
            if q is None:
                left[x] = 0.0
            else:
                left = torch.clamp(left - q, min=0.0)
                if case["drafts"] == "distinct":
                    q = q.clone()
                    q[x] = 0.0
                    q = q / q.sum() if float(q.sum()) > 0 else q
            if float(left.sum()) > 0:
                left = left / left.sum()
        if taken is not None:
            path.append(taken)
            continue
        if float(left.sum()) == 0:
            left = p
        upto = torch.cumsum(left, 0)
        over = (upto > float(s["v"][b].double()) * upto[-1]).nonzero()
        return path, int(over[0, 0]) if len(over) else case["vocab"] - 1


def exact(case, seed):
    s = prepare(case, seed)
    kind, docs, starts = case["kind"], s["docs"], s["starts"]
    if kind == "tree":
        depth, seen = [], []
        for _, parents in docs:
            depth += _depths(parents)
            seen += _bits(parents, _words(case))
        return _int32(depth), torch.tensor(seen, dtype=torch.int64).reshape(-1, _words(case)).to(DEV)
    if kind == "verify":
        path, kept, token = torch.full((len(docs), case["rows"]), -1, dtype=torch.int32), [0] * len(docs), [-1] * len(docs)
        u, tokens, parent = s["u"].double().tolist(), s["tokens"].tolist(), s["parent"].tolist()
        for b in range(len(docs)):
            if docs[b][1]:
                found, token[b] = _walk(s, b, range(starts[b], starts[b + 1]), s["target"], s["draft"], u, tokens, parent)
                path[b, :len(found)] = torch.tensor(found, dtype=torch.int32)
                kept[b] = len(found)
        return path.to(DEV), _int32(kept), _int32(token)
    ps, table = case["page"], s["pages"].cpu()
    if kind == "keep":
        out = [c.clone() for c in s["caches"]]
        for b, (c, path) in enumerate(docs):
            for i, r in enumerate(path):
                if i != r:
                    for new, old in zip(out, s["caches"]):
                        new[int(table[b, (c + i) // ps]), :, :, (c + i) % ps] = old[int(table[b, (c + r) // ps]), :, :, (c + r) % ps]
        return [x.double() for x in out]
    H, Hkv, dh, W, K = case["heads"], case["kv_heads"], case["d_head"], case["window"], case["sinks"]
    o = torch.zeros((starts[-1], H, dh), dtype=torch.float64, device=DEV)
    lse = torch.zeros((starts[-1], H), dtype=torch.float64, device=DEV)
    for b, (c, parents) in enumerate(docs):
        n = len(parents)
        if not n:
            continue
        depth = torch.tensor(_depths(parents), device=DEV)
        sees = torch.zeros((n, c + n), dtype=torch.bool)
        for i in range(n):                              # up to the root
            a = i
            while a >= 0:
                sees[i, c + a] = True
                a = parents[a]
        sees = sees.to(DEV)
        j = torch.arange(c, device=DEV)[None, :]
        sees[:, :c] = (c + depth[:, None] - j < W) | (j < K)
        held = torch.cat([s["cache"][int(table[b, i])].double() for i in range(-(-(c + n) // ps))], 2)[:, :, :c + n]
        q = s["qkv"][starts[b]:starts[b + 1]].double().reshape(n, H + 2 * Hkv, dh)
        for h in range(H):
            x = q[:, h] @ held[0, h // (H // Hkv)].T * float(dh) ** -0.5
            x = torch.where(sees, x, -math.inf)
            L = torch.logsumexp(x, 1)
            o[starts[b]:starts[b + 1], h] = torch.exp(x - L[:, None]) @ held[1, h // (H // Hkv)]
            lse[starts[b]:starts[b + 1], h] = L
    return o.reshape(starts[-1], -1), lse
