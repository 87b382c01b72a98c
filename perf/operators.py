"""Attention with a sliding window and sinks, forward and backward, and attention of new tokens over a paged cache, as
cases that can be timed.

`own` false: the operators in elementary torch operations, in 32 bits, rounded once at the end.  `own` true: the calls that a
program makes of `paper_2403_10616_amd`.  Sizes are those of the library's own configurations, or generic ones around them.

  window_fwd  row i of a document sees row j where j <= i and (j > i - window or j < sinks)
  window_bwd  its gradient, from o, lse and the gradient of o
  append      keys and values of new tokens into the pages of a cache
  paged       attention of the new tokens (a chunk each, or one token each) over the cache, with the same window and sinks
"""
import math
import random

import torch

own = False

DEV = "cuda"
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_ANY = 1 << 30                    # a window that reaches everything


def _window(name, kind, dtype, batch, seq, heads, kv_heads, d_head, window, sinks, ragged):
    return dict(name=name, kind=kind, dtype=dtype, batch=batch, seq=seq, heads=heads, kv_heads=kv_heads, d_head=d_head,
                window=window, sinks=sinks, ragged=ragged)


def _paged(name, kind, dtype, batch, new, cached, heads, kv_heads, d_head, page, window, sinks, ragged):
    return dict(name=name, kind=kind, dtype=dtype, batch=batch, new=new, cached=cached, heads=heads, kv_heads=kv_heads,
                d_head=d_head, page=page, window=window, sinks=sinks, ragged=ragged)


def listed():
    return [
        # The smoke-size path in fp32, four sequences of 64: a parity run.  Latency.
        _window("window forward tiny fp32", "window_fwd", "f32", 4, 64, 2, 2, 32, 16, 2, False),
        # A block of the 150M path at the round's 16 x 2048 tokens, trained with a window of 512.
        _window("window forward 150M", "window_fwd", "bf16", 16, 2048, 14, 14, 64, 512, 4, False),
        # Two long documents under a path whose heads share keys: prefill or scoring of whole texts, padded to the longer one.
        _window("window forward long shared heads", "window_fwd", "bf16", 2, 32768, 16, 4, 128, 4096, 64, True),
        # The gradient of the 150M block.
        _window("window backward 150M", "window_bwd", "bf16", 16, 2048, 14, 14, 64, 512, 4, False),
        # A padded batch of a small path trained in fp32.
        _window("window backward fp32 ragged", "window_bwd", "f32", 8, 500, 8, 8, 64, 100, 1, True),
        # Training on long documents, wide heads that share keys, lengths apart.
        _window("window backward shared heads", "window_bwd", "bf16", 4, 8000, 16, 4, 128, 1000, 16, True),
        # A serving batch: one new token for each of 64 documents of the 150M path.  Latency.
        _paged("append one token each", "append", "bf16", 64, 1, 1500, 14, 14, 64, 16, _ANY, 0, True),
        # Prefill of eight documents in chunks.
        _paged("append chunks", "append", "bf16", 8, 2000, 3000, 16, 8, 128, 64, _ANY, 0, True),
        # One document of the 150M path is being continued.  Latency.
        _paged("paged one token", "paged", "bf16", 1, 1, 1000, 14, 14, 64, 16, _ANY, 0, False),
        # A serving batch over long caches of every length.
        _paged("paged tokens long", "paged", "bf16", 64, 1, 16000, 16, 4, 128, 64, _ANY, 0, True),
        # The next chunks of four long documents, under the window that the path was trained with.
        _paged("paged chunks window", "paged", "bf16", 4, 512, 12000, 14, 14, 64, 16, 2048, 4, True),
        # A small path in fp32, chunks of up to forty tokens: evaluation that re-routes between chunks.
        _paged("paged chunks fp32", "paged", "f32", 5, 40, 700, 8, 2, 32, 32, _ANY, 0, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_MOST_FLOPS, _MOST_BYTES = 1.6e12, 5.9e8      # the largest listed cases


def draw(rng):
    while True:
        kind = rng.choice(("window_fwd", "window_bwd", "append", "paged", "paged"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        d_head = rng.choice((32, 64, 64, 128))
        kv = _log_int(rng, 1, 16)
        heads = kv * rng.choice((1, 1, 2, 3, 4, 8))
        window = rng.choice((_ANY, _log_int(rng, 1, 4096), _log_int(rng, 16, 4096)))
        sinks = rng.choice((0, _log_int(rng, 1, 128)))
        ragged = rng.random() < 0.6
        if kind.startswith("window"):
            case = _window(None, kind, dtype, _log_int(rng, 1, 32), _log_int(rng, 1, 16000), heads, kv, d_head, window, sinks, ragged)
        else:
            new = 1 if rng.random() < 0.5 else _log_int(rng, 2, 2000)
            case = _paged(None, kind, dtype, _log_int(rng, 1, 128), new, rng.choice((0, _log_int(rng, 1, 30000), _log_int(rng, 1, 30000))),
                          heads, kv, d_head, rng.choice((16, 32, 64, 128)), window, sinks, ragged)
        del case["name"]
        w = work(case)
        # the fp32 matrix cores are a sixteenth as fast as the bf16 ones
        if heads <= 32 and w["flops"] * (16 if dtype == "f32" else 1) <= _MOST_FLOPS and w["bytes"] <= _MOST_BYTES \
                and _cache_bytes(case) <= 8.0e8:
            return case


# ---- lengths: a case's own, whatever the seed of its data ----------------------------------------------------------
def _lengths(case):
    """window_*: rows of each document.  append, paged: (cached positions, new tokens) of each document."""
    B, rng = case["batch"], random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    if case["kind"].startswith("window"):
        S = case["seq"]
        return [S] + [rng.randint(max(1, S // 4), S) if case["ragged"] else S for _ in range(B - 1)]
    if not case["ragged"]:
        return [(case["cached"], case["new"])] * B
    return [(case["cached"], case["new"])] + [(rng.randint(0, case["cached"]), rng.randint(min(1, case["new"] - 1), case["new"]))
                                             for _ in range(B - 1)]


def _cache_bytes(case):
    if case["kind"].startswith("window"):
        return 0
    ps = case["page"]
    return sum(-(-(c + n) // ps) for c, n in _lengths(case)) * ps * 2 * case["kv_heads"] * case["d_head"] * (4 if case["dtype"] == "f32" else 2)


def _visible(i, window, sinks):
    """how many rows row i sees"""
    near = min(window, i + 1)
    return near + min(sinks, i + 1 - near)


def _pairs(first, n, window, sinks):
    """sum of _visible over rows first .. first + n - 1; constant from row window + sinks on"""
    total, i, end = 0, first, first + n
    while i < end and i < window + sinks:
        if i + 1 <= window:                       # all rows up to here see everything before them
            upto = min(end, window)
            total += (i + 1 + upto) * (upto - i) // 2
            i = upto
        else:                                     # the window is full, the sinks are not
            upto = min(end, window + sinks)
            total += (upto - i) * window + (i + 1 - window + upto - window) * (upto - i) // 2
            i = upto
    return total + (end - i) * _visible(max(i, window + sinks), window, sinks) if i < end else total


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    H, Hkv, dh, W, K = case["heads"], case["kv_heads"], case["d_head"], case["window"], case["sinks"]
    lens = _lengths(case)
    if case["kind"].startswith("window"):
        rows, padded = sum(lens), case["batch"] * case["seq"]
        pairs = sum(_pairs(0, n, W, K) for n in lens)
        if case["kind"] == "window_fwd":
            return dict(bytes=rows * (H + 2 * Hkv) * dh * es + padded * H * (dh * es + 4), flops=4.0 * dh * H * pairs)
        return dict(bytes=rows * ((3 * H + 2 * Hkv) * dh * es + 4 * H) + padded * (H + 2 * Hkv) * dh * es, flops=10.0 * dh * H * pairs)
    rows = sum(n for _, n in lens)
    if case["kind"] == "append":
        return dict(bytes=rows * 4 * Hkv * dh * es, flops=0.0)
    seen = 0
    for c, n in lens:                              # positions that some new token of the document sees
        if n:
            first = max(0, c - W + 1)
            seen += c + n - first + min(K, first)
    pairs = sum(_pairs(c, n, W, K) for c, n in lens)
    return dict(bytes=seen * 2 * Hkv * dh * es + rows * H * (2 * dh * es + 4), flops=4.0 * dh * H * pairs)


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(shape, device=DEV, generator=g)


def _projected(g, rows, H, Hkv, dh, dtype):
    """rows of q | k | v: a LayerNorm's output through the projection, keys with a common part, values smaller"""
    x = _randn(g, rows, (H + 2 * Hkv) * dh)
    x[:, :H * dh] *= 1.5
    x[:, H * dh:(H + Hkv) * dh] += 0.5 * _randn(g, 1, Hkv * dh)
    x[:, (H + Hkv) * dh:] *= 0.5
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    t, H, Hkv, dh = _TYPES[case["dtype"]], case["heads"], case["kv_heads"], case["d_head"]
    s = dict(case=case, lens=_lengths(case))
    if case["kind"].startswith("window"):
        B, S = case["batch"], case["seq"]
        s["qkv"] = _projected(g, B * S, H, Hkv, dh, t)
        s["lengths"] = torch.tensor(s["lens"], dtype=torch.int32, device=DEV) if case["ragged"] else None
        if case["kind"] == "window_fwd":
            s["o"] = torch.empty((B * S, H * dh), dtype=t, device=DEV)
            s["lse"] = torch.empty((B, H, S), device=DEV)
        else:                                      # what the forward pass left, and the gradient of the layers above
            s["o"], s["lse"] = _plain_window_fwd(s)
            s["d_o"] = _randn(g, B * S, H * dh).to(t)
            s["dqkv"] = torch.empty_like(s["qkv"])
            s["dsum"] = torch.empty(2 * B * H * (-(-S // 128) * 128), device=DEV)
        return s
    ps, lens = case["page"], s["lens"]
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    s["starts"] = starts
    used = [-(-(c + n) // ps) for c, n in lens]
    per_doc, n_pages = max(used) + 1, sum(used) + 3
    order = torch.randperm(n_pages, device=DEV, generator=g).tolist()
    table = torch.full((len(lens), per_doc), -1, dtype=torch.int32)
    for b, n in enumerate(used):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    s["pages"], s["n_pages"], s["per_doc"] = table.to(DEV), n_pages, per_doc
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["cache_len"] = torch.tensor([c for c, _ in lens], dtype=torch.int32, device=DEV)
    s["qkv"] = _projected(g, starts[-1], H, Hkv, dh, t)
    # a cache that holds tokens of the same kind as the new ones
    cache = _randn(g, n_pages, 2, Hkv, ps, dh)
    cache[:, 0] += 0.5 * _randn(g, 1, Hkv, 1, dh)
    cache[:, 1] *= 0.5
    s["cache"] = cache.to(t)
    del cache
    if case["kind"] == "paged":
        _plain_append(s)
        s["o"] = torch.empty((starts[-1], H * dh), dtype=t, device=DEV)
        s["lse"] = torch.empty((starts[-1], H), device=DEV)
        if own:
            import paper_2403_10616_amd as dp
            n = dp.dipaco_k_attention_paged_workspace_bytes(starts[-1], len(lens), case["new"], H, Hkv, dh, ps, per_doc)
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------
_ROWS = 512                       # query rows taken at a time: the scores of a block are written down


def _split(x, H, Hkv, dh):
    """[heads, rows, dh] in 32 bits"""
    x = x.float()
    q, k, v = x[:, :H * dh], x[:, H * dh:(H + Hkv) * dh], x[:, (H + Hkv) * dh:]
    return [p.reshape(p.shape[0], -1, dh).transpose(0, 1).contiguous() for p in (q, k, v)]


def _blocks(first, n, window, sinks):
    """(rows of a block, the keys that any of them sees, which row sees which key) over rows first .. first + n - 1"""
    for lo in range(first, first + n, _ROWS):
        hi = min(first + n, lo + _ROWS)
        near = max(0, lo - window + 1)
        keys = torch.cat([torch.arange(0, min(sinks, near), device=DEV), torch.arange(near, hi, device=DEV)])
        i, j = torch.arange(lo, hi, device=DEV)[:, None], keys[None, :]
        yield slice(lo - first, hi - first), keys, (j <= i) & ((j > i - window) | (j < sinks))


def _scores(q, k, sees, G, dh):
    """[heads, rows, keys]; the heads of a group share k"""
    Hkv = k.shape[0]
    s = torch.matmul(q.reshape(Hkv, -1, dh), k.transpose(1, 2)).reshape(Hkv * G, q.shape[1], -1) / math.sqrt(dh)
    return s.masked_fill_(~sees, -math.inf)


def _attend(q, k, v, first, case):
    """o [heads, rows, dh] and lse [heads, rows] of rows first .. of a document whose keys and values are k, v"""
    H, n, dh = q.shape
    Hkv, G = k.shape[0], H // k.shape[0]
    o, lse = torch.empty_like(q), torch.empty((H, n), device=DEV)
    for rows, keys, sees in _blocks(first, n, case["window"], case["sinks"]):
        s = _scores(q[:, rows], k[:, keys], sees, G, dh)
        top = s.amax(2, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(2, keepdim=True)
        o[:, rows] = (torch.matmul(p.reshape(Hkv, -1, p.shape[2]), v[:, keys]).reshape(H, -1, dh)) / total
        lse[:, rows] = (top + torch.log(total))[:, :, 0]
    return o, lse


def _plain_window_fwd(s):
    case, S, H = s["case"], s["case"]["seq"], s["case"]["heads"]
    o = torch.zeros((len(s["lens"]) * S, H * case["d_head"]), dtype=s["qkv"].dtype, device=DEV)
    lse = torch.zeros((len(s["lens"]), H, S), device=DEV)
    for b, n in enumerate(s["lens"]):
        q, k, v = _split(s["qkv"][b * S:b * S + n], H, case["kv_heads"], case["d_head"])
        ob, lse[b, :, :n] = _attend(q, k, v, 0, case)
        o[b * S:b * S + n] = ob.transpose(0, 1).reshape(n, -1).to(o.dtype)
    return o, lse


def _plain_window_bwd(s):
    case, S, H, Hkv, dh = s["case"], s["case"]["seq"], s["case"]["heads"], s["case"]["kv_heads"], s["case"]["d_head"]
    G, scale = H // Hkv, 1.0 / math.sqrt(dh)
    out = torch.zeros_like(s["qkv"])
    for b, n in enumerate(s["lens"]):
        at = slice(b * S, b * S + n)
        q, k, v = _split(s["qkv"][at], H, Hkv, dh)
        g, o = (s[x][at].float().reshape(n, H, dh).transpose(0, 1).contiguous() for x in ("d_o", "o"))
        D = (g * o).sum(2, keepdim=True)
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
        for rows, keys, sees in _blocks(0, n, case["window"], case["sinks"]):
            gr, qr = g[:, rows].reshape(Hkv, -1, dh), q[:, rows].reshape(Hkv, -1, dh)
            p = torch.exp(_scores(q[:, rows], k[:, keys], sees, G, dh) - s["lse"][b, :, rows, None])
            dp = torch.matmul(gr, v[:, keys].transpose(1, 2)).reshape(p.shape)
            ds = (p * (dp - D[:, rows])).reshape(Hkv, -1, len(keys))
            dq[:, rows] = torch.matmul(ds, k[:, keys]).reshape(H, -1, dh) * scale
            dk.index_add_(1, keys, torch.matmul(ds.transpose(1, 2), qr) * scale)
            dv.index_add_(1, keys, torch.matmul(p.reshape(Hkv, -1, len(keys)).transpose(1, 2), gr))
        out[at] = torch.cat([x.transpose(0, 1).reshape(n, -1) for x in (dq, dk, dv)], 1).to(out.dtype)
    return out


def _places(s, b, lo, hi):
    """pages and slots of positions lo .. hi - 1 of document b"""
    p = torch.arange(lo, hi, device=DEV)
    return s["pages"][b][p // s["case"]["page"]].long(), p % s["case"]["page"]


def _plain_append(s):
    case = s["case"]
    H, Hkv, dh = case["heads"], case["kv_heads"], case["d_head"]
    for b, (c, n) in enumerate(s["lens"]):
        if n:
            kv = s["qkv"][s["starts"][b]:s["starts"][b + 1], H * dh:].reshape(n, 2, Hkv, dh)
            page, slot = _places(s, b, c, c + n)
            s["cache"][page, :, :, slot] = kv
    return s["cache"]


def _plain_paged(s):
    case = s["case"]
    H, Hkv, dh = case["heads"], case["kv_heads"], case["d_head"]
    o = torch.zeros((s["starts"][-1], H * dh), dtype=s["qkv"].dtype, device=DEV)
    lse = torch.zeros((s["starts"][-1], H), device=DEV)
    for b, (c, n) in enumerate(s["lens"]):
        if n:
            at = slice(s["starts"][b], s["starts"][b + 1])
            page, slot = _places(s, b, 0, c + n)
            kv = s["cache"][page, :, :, slot].float()          # [positions, 2, Hkv, dh]
            k, v = (kv[:, x].transpose(0, 1).contiguous() for x in (0, 1))
            q = s["qkv"][at, :H * dh].float().reshape(n, H, dh).transpose(0, 1).contiguous()
            ob, lb = _attend(q, k, v, c, case)
            o[at], lse[at] = ob.transpose(0, 1).reshape(n, -1).to(o.dtype), lb.transpose(0, 1)
    return o, lse


_PLAIN = dict(window_fwd=_plain_window_fwd, window_bwd=_plain_window_bwd, append=_plain_append, paged=_plain_paged)


# ---- the calls a program makes --------------------------------------------------------------------------------------
def _own(s):
    import paper_2403_10616_amd as dp
    case, kind = s["case"], s["case"]["kind"]
    dtype = dp.F32 if case["dtype"] == "f32" else dp.BF16
    H, Hkv, dh, W, K = case["heads"], case["kv_heads"], case["d_head"], case["window"], case["sinks"]
    if kind == "window_fwd":
        dp.dipaco_k_attention_window_fwd(dtype, s["qkv"], s["lengths"], s["o"], s["lse"], case["batch"], case["seq"], H, Hkv, dh, W, K)
        return s["o"], s["lse"]
    if kind == "window_bwd":
        dp.dipaco_k_attention_window_bwd(dtype, s["qkv"], s["lengths"], s["o"], s["d_o"], s["lse"], s["dqkv"], s["dsum"], case["batch"],
                                         case["seq"], H, Hkv, dh, W, K)
        return s["dqkv"]
    T, B = s["starts"][-1], len(s["lens"])
    if kind == "append":
        dp.dipaco_k_cache_append(dtype, s["qkv"], s["row_start"], s["cache_len"], s["pages"], s["cache"], T, B, H, Hkv, dh,
                                 s["n_pages"], case["page"], s["per_doc"])
        return s["cache"]
    dp.dipaco_k_attention_paged(dtype, s["qkv"], s["row_start"], s["cache_len"], s["pages"], s["cache"], s["o"], s["lse"], T, B,
                                case["new"], H, Hkv, dh, s["n_pages"], case["page"], s["per_doc"], W, K, s["ws"])
    return s["o"], s["lse"]


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["kind"]](state)


# ---- the definition in 64 bits: a head at a time, every pair of a block of rows written down, seen or not -----------------
_EXACT_PAIRS = 40e9               # pairs (rows x all keys before the last) that take a few seconds


def _seen(rows, keys, window, sinks):
    ahead = keys[None, :] > rows[:, None]
    far = (rows[:, None] - keys[None, :] >= window) & (keys[None, :] >= sinks)
    return ~(ahead | far)


def _exact_head(q, k, v, first, window, sinks, per):
    """per(rows, P, s) for each block of rows; q [n, dh], k and v [m, dh] in 64 bits"""
    keys, step = torch.arange(k.shape[0], device=DEV), max(16, int(5e7 // max(1, k.shape[0])))
    for lo in range(0, q.shape[0], step):
        rows = slice(lo, min(q.shape[0], lo + step))
        at = first + torch.arange(rows.start, rows.stop, device=DEV)
        s = (q[rows] @ k.T) * dh_scale(q.shape[1])
        per(rows, _seen(at, keys, window, sinks), s)


def dh_scale(dh):
    return float(dh) ** -0.5


def exact(case, seed):
    s = prepare(case, seed)
    kind, H, Hkv, dh, W, K = case["kind"], case["heads"], case["kv_heads"], case["d_head"], case["window"], case["sinks"]
    G = H // Hkv
    if kind == "append":
        out = s["cache"].double()
        ps = case["page"]
        table = s["pages"].cpu()
        for b, (c, n) in enumerate(s["lens"]):
            done = 0
            while done < n:                       # page by page
                slot = (c + done) % ps
                take = min(ps - slot, n - done)
                rows = s["qkv"][s["starts"][b] + done:s["starts"][b] + done + take].double()
                kv = rows[:, H * dh:].reshape(take, 2, Hkv, dh)
                out[int(table[b, (c + done) // ps]), :, :, slot:slot + take] = kv.permute(1, 2, 0, 3)
                done += take
        return out
    lens = s["lens"]
    m_of = [(0, n) for n in lens] if kind.startswith("window") else lens
    if H * sum(n * (c + n) for c, n in m_of) > _EXACT_PAIRS:
        return None
    qkv = s["qkv"].double()
    T = qkv.shape[0]
    o = torch.zeros((T, H, dh), dtype=torch.float64, device=DEV)
    L = torch.zeros((T, H), dtype=torch.float64, device=DEV)
    grad = torch.zeros((T, H + 2 * Hkv, dh), dtype=torch.float64, device=DEV)
    table = None if kind.startswith("window") else s["pages"].cpu()
    for b, (c, n) in enumerate(m_of):
        if not n:
            continue
        r0 = b * case["seq"] if kind.startswith("window") else s["starts"][b]
        mine = qkv[r0:r0 + n].reshape(n, H + 2 * Hkv, dh)
        if kind == "paged":
            ps = case["page"]
            held = torch.cat([s["cache"][int(table[b, i])].double() for i in range(-(-(c + n) // ps))], 2)[:, :, :c + n]
            keys, values = held[0], held[1]       # [Hkv, positions, dh]
        else:
            keys, values = mine[:, H:H + Hkv].transpose(0, 1), mine[:, H + Hkv:].transpose(0, 1)
        for h in range(H):
            k, v, q = keys[h // G], values[h // G], mine[:, h]
            if kind == "window_bwd":
                go = s["d_o"][r0:r0 + n].double().reshape(n, H, dh)[:, h]
                D = (go * s["o"][r0:r0 + n].double().reshape(n, H, dh)[:, h]).sum(1)
                given = s["lse"][b, h].double()

                def per(rows, sees, sc):
                    P = torch.where(sees, torch.exp(sc - given[rows][:, None]), 0.0)
                    dS = P * (go[rows] @ v.T - D[rows][:, None])
                    grad[r0 + rows.start:r0 + rows.stop, h] = dS @ k * dh_scale(dh)
                    grad[r0:r0 + n, H + h // G] += dS.T @ q[rows] * dh_scale(dh)
                    grad[r0:r0 + n, H + Hkv + h // G] += P.T @ go[rows]
            else:
                def per(rows, sees, sc):
                    sc = torch.where(sees, sc, -math.inf)
                    lse = torch.logsumexp(sc, 1)
                    o[r0 + rows.start:r0 + rows.stop, h] = torch.exp(sc - lse[:, None]) @ v
                    L[r0 + rows.start:r0 + rows.stop, h] = lse
            _exact_head(q, k, v, c, W, K, per)
    if kind == "window_bwd":
        return grad.reshape(T, -1)
    o = o.reshape(T, -1)
    if kind == "paged":
        return o, L
    return o, L.reshape(case["batch"], case["seq"], H).transpose(1, 2).contiguous()
