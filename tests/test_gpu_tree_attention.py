"""Attention of trees of drafted tokens over a paged cache, against the definition in 64 bits, and a whole step of drafted decoding."""
import math
import random

import pytest
import torch

import attention_reference as aref
import draft_reference as ref
import paper_2403_10616_amd as dp
from gpu_util import DEV
from test_gpu_drafts import tree, verify
from test_gpu_paged import Cache, guarded_workspace, i32, starts_of
from test_gpu_window import ALL, TDT, draw, heads_of

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
INF = math.inf


def attend(c, qkv, starts, lens, depth, seen, H, max_new, window, sinks, rows=None, want_lse=True, ws=None):
    T, B = starts[-1] if rows is None else rows, len(lens)
    o = torch.full((T, H * c.dh), 77.0, dtype=TDT[c.dtype], device=DEV)
    lse = torch.full((T, H), 77.0, device=DEV) if want_lse else None
    if ws is None:
        ws = torch.full((dp.dipaco_k_attention_tree_workspace_bytes(T, B, max_new, H, c.Hkv, c.dh, c.page, c.per_doc),), 255, dtype=torch.uint8, device=DEV)
    dp.dipaco_k_attention_tree(c.dtype, qkv, i32(starts), i32(lens), depth, seen, c.pages, c.data, o, lse, T, B, max_new, H, c.Hkv, c.dh, c.n_pages, c.page,
                               c.per_doc, window, sinks, ws)
    return o, lse


def mask_of(cached, rows_seen, depths, window, sinks, positions):
    """[rows, positions]: which row sees which position"""
    n = len(rows_seen)
    m = torch.zeros((n, max(positions, cached + n)), dtype=torch.bool)
    for i in range(n):
        j = torch.arange(cached)
        m[i, :cached] = (j > cached + depths[i] - window) | (j < sinks)
        m[i, [cached + a for a in rows_seen[i] if a < n]] = True
    return m[:, :positions]


def filled(dtype, cached, counts, H, Hkv, dh, page, seed, scale=1.0):
    """a cache that holds `cached` positions and the new rows of each document, and the rows"""
    c = Cache(dtype, [a + b for a, b in zip(cached, counts)], Hkv, dh, page, seed)
    if any(cached):
        st = starts_of(cached)
        c.append(draw((st[-1], (H + 2 * Hkv) * dh), seed, dtype).to(DEV), st, [0] * len(cached), H)
    st = starts_of(counts)
    x = draw((st[-1], (H + 2 * Hkv) * dh), seed + 1, dtype, scale)
    c.append(x.to(DEV), st, cached, H)
    return c, x, st


def check(dtype, cached, counts, shape, H, Hkv, dh, page, window, sinks, seed=3, scale=1.0, max_new=None):
    print(f"tree dtype={dtype} cached={cached} rows={counts} {shape} H={H} Hkv={Hkv} dh={dh} page={page} W={window} sinks={sinks}", flush=True)
    rng = random.Random(seed)
    c, x, st = filled(dtype, cached, counts, H, Hkv, dh, page, seed, scale)
    n = max(counts) if max_new is None else max_new
    parents = [ref.random_parents(rng, k, shape) for k in counts]
    depth, seen = tree(parents, max_new=n)
    o, lse = attend(c, x.to(DEV), st, cached, depth, seen, H, n, window, sinks)
    for b, (m, k) in enumerate(zip(cached, counts)):
        if k:
            rows = ref.seen_rows(parents[b])
            mask = mask_of(m, rows, [len(r) - 1 for r in rows], window, sinks, m + k)
            kv = c.kv[b].double()
            q = heads_of(x[st[b]:st[b + 1]], k, H, Hkv, dh)[0]
            wo, wl, eo, el = aref.forward(q, kv[:, 0], kv[:, 1], mask, TDT[dtype])
            aref.inside(o[st[b]:st[b + 1]].reshape(k, H, dh), wo, eo, f"o[{b}]")
            aref.inside(lse[st[b]:st[b + 1]], wl, el, f"lse[{b}]")
    o2, lse2 = attend(c, x.to(DEV), st, cached, depth, seen, H, n, window, sinks)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    o3, _ = attend(c, x.to(DEV), st, cached, depth, seen, H, n, window, sinks, want_lse=False)
    assert torch.equal(o, o3)


@TYPES
@pytest.mark.parametrize("dh,page", [(32, 16), (64, 16), (64, 64), (128, 32), (128, 256), (64, 128)])
@pytest.mark.parametrize("cached,counts,shape,H,Hkv,window,sinks", [
    ([0], [1], "chain", 1, 1, ALL, 0), ([0, 0], [7, 33], "level", 2, 2, ALL, 0), ([63, 64, 65, 0], [5, 6, 1, 8], "deep", 2, 2, ALL, 0),
    ([500, 3], [16, 12], "forest", 8, 2, 100, 4), ([700, 129], [9, 0], "level", 16, 1, ALL, 0), ([0, 30], [70, 1], "chain", 4, 2, 70, 2),
    ([300, 0, 5], [40, 33, 128], "level", 3, 1, 128, 0), ([1000], [5], "star", 6, 2, 5, 0), ([90, 257], [17, 64], "deep", 8, 8, 70, 70),
    ([31, 40], [65, 130], "forest", 2, 1, ALL, 0)])
def test_trees_over_a_cache(dtype, dh, page, cached, counts, shape, H, Hkv, window, sinks):
    check(dtype, cached, counts, shape, H, Hkv, dh, page, window, sinks)


@TYPES
@pytest.mark.parametrize("cached,counts,shape,H,Hkv,dh,page,window,sinks", [
    ([9000], [16], "level", 2, 1, 64, 64, ALL, 0), ([9000, 10], [5, 7], "deep", 4, 1, 128, 16, 5000, 100), ([6000], [40], "level", 4, 2, 32, 32, ALL, 0),
    ([3000, 0], [200, 1], "deep", 2, 2, 64, 16, 1500, 3), ([5000, 2500, 1, 0, 777], [8] * 5, "level", 6, 2, 64, 16, ALL, 0),
    ([2000, 3000], [500, 400], "level", 4, 2, 64, 16, 600, 4), ([700], [1024], "forest", 2, 1, 64, 32, 1024, 0), ([6000, 2000, 50], [1, 300, 400], "deep", 8, 1, 64, 64, ALL, 0)])
def test_long_caches_and_large_trees(dtype, cached, counts, shape, H, Hkv, dh, page, window, sinks):
    check(dtype, cached, counts, shape, H, Hkv, dh, page, window, sinks, seed=6)


def lengths(seed, n, most):
    """documents of lengths apart: most of them short, a few of `most`, some empty"""
    rng = random.Random(seed)
    return [rng.choice([0, rng.randint(0, 200), rng.randint(0, most), most]) for _ in range(n)]


@TYPES
@pytest.mark.parametrize("cached,counts,H,Hkv,dh,page,window,sinks", [
    ([5000, 10], [40, 70], 2, 1, 32, 16, ALL, 0), ([0, 9000, 30, 4500], [64, 33, 0, 200], 4, 2, 64, 64, ALL, 0), ([20000, 5], [64, 64], 4, 4, 32, 32, ALL, 0),
    ([6000, 5900, 6100], [150, 1, 90], 2, 2, 128, 64, 5000, 70), (lengths(1, 64, 4200), [36] * 64, 2, 1, 32, 64, ALL, 0),
    (lengths(2, 65, 4200), [36] * 65, 2, 1, 32, 64, ALL, 0), (lengths(3, 30, 4300), [k % 45 for k in range(30)], 16, 16, 32, 16, ALL, 3),
    ([4200, 4200], [1024, 1000], 1, 1, 64, 32, ALL, 0), ([4500] * 5, [9, 10, 33, 34, 8], 8, 2, 128, 32, ALL, 0)])
def test_long_documents_of_lengths_apart(dtype, cached, counts, H, Hkv, dh, page, window, sinks):
    """splits of equal length for all documents: one document far longer than the others, as many documents as a wave has lanes and one more,
    documents without rows, with few rows and with several blocks of them"""
    check(dtype, cached, counts, "level", H, Hkv, dh, page, window, sinks, seed=12)


def test_long_documents_that_have_outgrown_their_table_or_lost_pages():
    dtype, H, Hkv, dh, page = dp.BF16, 4, 2, 64, 64
    cached, counts = [4400, 4400, 100, 4000], [60, 50, 70, 64]
    c, x, st = filled(dtype, cached, counts, H, Hkv, dh, page, 5)
    for b, gone in enumerate([range(10, 50), range(0, c.per_doc), [0], [60, 62]]):
        for at in gone:
            if c.table[b][at] >= 0:
                c.data[c.table[b][at]] = float("nan")
            c.table[b][at] = -1
    c.pages = i32(c.table)
    depth, seen = tree([ref.random_parents(random.Random(b), k, "deep") for b, k in enumerate(counts)])
    lens = [4400, 4400, 100, 1 << 29]                            # the last one's rows see none of its table, nor each other
    parents = [ref.random_parents(random.Random(b), k, "deep") for b, k in enumerate(counts)]
    o, lse = attend(c, x.to(DEV), st, lens, depth, seen, H, max(counts), 4200, 0)
    for b, (m, k) in enumerate(zip(cached, counts)):
        at = slice(st[b], st[b + 1])
        if b == 3:
            assert not o[at].any() and bool((lse[at] == -INF).all())
            continue
        rows = ref.seen_rows(parents[b])
        held = torch.tensor([c.table[b][p // page] >= 0 for p in range(m + k)])
        mask = mask_of(m, rows, [len(r) - 1 for r in rows], 4200, 0, m + k) & held
        kv, q = c.kv[b].double(), heads_of(x[at], k, H, Hkv, dh)[0]
        wo, wl = aref.definition(q, kv[:, 0], kv[:, 1], mask)
        _, _, eo, el = aref.forward(q, kv[:, 0], kv[:, 1], mask, TDT[dtype])
        aref.inside(o[at].reshape(k, H, dh), wo, eo, f"o[{b}]")
        aref.inside(lse[at], wl, el.nan_to_num(), f"lse[{b}]")


@TYPES
def test_peaked_rows(dtype):
    check(dtype, [400, 30], [30, 3], "level", 4, 2, 64, 16, ALL, 0, seed=8, scale=8.0)


@TYPES
def test_many_documents(dtype):
    rng = random.Random(5)
    check(dtype, [rng.randint(0, 90) for _ in range(150)], [rng.randint(0, 9) for _ in range(150)], "level", 2, 1, 32, 16, 40, 2, seed=9, max_new=12)


@TYPES
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("cached,counts", [([40, 0, 3], [20, 9, 33]), ([0, 200], [70, 150])])
def test_any_bits(dtype, dh, cached, counts):
    """rows that see later rows, none, or rows that the document does not have; depths outside their range are taken as the nearest inside"""
    H, Hkv, page, window, sinks = 4, 2, 16, 160, 1
    c, x, st = filled(dtype, cached, counts, H, Hkv, dh, page, 11)
    rng, n, T = random.Random(4), max(counts), st[-1]
    words = -(-n // 64)
    rows, bits, depth = [], [], []
    for b, k in enumerate(counts):
        for i in range(k):
            r = frozenset(a for a in range(64 * words) if rng.random() < 0.3) if i % 4 else frozenset()
            rows.append(r)
            bits.append(ref.words_of(r, words))
            depth.append(rng.choice([0, i, i // 2, -3, 1 << 30]))
    o, lse = attend(c, x.to(DEV), st, cached, i32(depth), torch.tensor(bits, dtype=torch.int64, device=DEV), H, n, window, sinks)
    for b, (m, k) in enumerate(zip(cached, counts)):
        at = slice(st[b], st[b + 1])
        mask = mask_of(m, rows[at], [min(max(d, 0), i) for i, d in enumerate(depth[at])], window, sinks, m + k)
        kv = c.kv[b].double()
        q = heads_of(x[at], k, H, Hkv, dh)[0]
        wo, wl = aref.definition(q, kv[:, 0], kv[:, 1], mask)
        _, _, eo, el = aref.forward(q, kv[:, 0], kv[:, 1], mask, TDT[dtype])
        assert m > 0 or bool((wl == -INF).any())                    # rows that see nothing are among them
        aref.inside(o[at].reshape(k, H, dh), wo, eo, f"o[{b}]")
        aref.inside(lse[at], wl, el.nan_to_num(), f"lse[{b}]")


@TYPES
@pytest.mark.parametrize("counts", [[5, 9, 6], [40, 33, 70]])
def test_pages_that_are_gone_hold_no_keys(dtype, counts):
    """holes among the cached positions and under the drafted rows, a document without pages, entries beyond the pages; what the table does
    not name holds NaN"""
    H, Hkv, dh, page, cached = 4, 2, 64, 16, [100, 100, 60]
    c, x, st = filled(dtype, cached, counts, H, Hkv, dh, page, 2)
    for b, gone in enumerate([range(2, 4), range(0, c.per_doc), [0, (60 + counts[2] - 1) // page]]):
        for at in gone:
            if 0 <= c.table[b][at] < c.n_pages:
                c.data[c.table[b][at]] = float("nan")
            c.table[b][at] = [-1, c.n_pages, -(1 << 31), (1 << 31) - 1][at % 4]
    c.pages = i32(c.table)
    parents = [ref.random_parents(random.Random(7), k, "level") for k in counts]
    n = max(counts)
    depth, seen = tree(parents)
    o, lse = attend(c, x.to(DEV), st, cached, depth, seen, H, n, ALL, 0)
    for b, (m, k) in enumerate(zip(cached, counts)):
        rows = ref.seen_rows(parents[b])
        held = torch.tensor([0 <= c.table[b][p // page] < c.n_pages for p in range(m + k)])
        mask = mask_of(m, rows, [len(r) - 1 for r in rows], ALL, 0, m + k) & held
        kv, q = c.kv[b].double(), heads_of(x[st[b]:st[b + 1]], k, H, Hkv, dh)[0]
        wo, wl = aref.definition(q, kv[:, 0], kv[:, 1], mask)
        _, _, eo, el = aref.forward(q, kv[:, 0], kv[:, 1], mask, TDT[dtype])
        aref.inside(o[st[b]:st[b + 1]].reshape(k, H, dh), wo, eo, f"o[{b}]")
        aref.inside(lse[st[b]:st[b + 1]], wl, el.nan_to_num(), f"lse[{b}]")


@TYPES
@pytest.mark.parametrize("dh,page", [(32, 16), (64, 32), (128, 16)])
@pytest.mark.parametrize("cached,counts,window,sinks", [([70, 64, 60], [3, 30, 30], 40, 2), ([50, 0, 64], [40, 5, 1], ALL, 0), ([50, 10], [100, 90], 120, 0),
                                                        ([1 << 30, (1 << 28) + 7, 63], [2, 33, 9], ALL, 0), ([(1 << 30) - 5, 62, 1 << 30], [9, 3, 40], 70, 5)])
def test_documents_that_have_outgrown_their_table(dtype, dh, page, cached, counts, window, sinks):
    """64 positions a table: rows keep their positions, and see what of the table they would see"""
    print(f"outgrown dtype={dtype} cached={cached} rows={counts} dh={dh} page={page} W={window} sinks={sinks}", flush=True)
    room, B, H, Hkv = 64, len(cached), 4, 2
    c = Cache(dtype, [room] * B, Hkv, dh, page, 3)
    data = draw(tuple(c.data.shape), 5, dtype)
    c.data.copy_(data)
    st = starts_of(counts)
    x = draw((st[-1], (H + 2 * Hkv) * dh), 6, dtype)
    parents = [ref.random_parents(random.Random(b), k, "level") for b, k in enumerate(counts)]
    depth, seen = tree(parents)
    o, lse = attend(c, x.to(DEV), st, cached, depth, seen, H, max(counts), window, sinks)
    for b, (m, k) in enumerate(zip(cached, counts)):
        rows = ref.seen_rows(parents[b])
        kv = torch.cat([data[p] for p in c.table[b]], 2).double().permute(2, 0, 1, 3)
        mask = torch.zeros((k, room), dtype=torch.bool)
        for i in range(k):
            for j in range(room):
                mask[i, j] = j > m + len(rows[i]) - 1 - window or j < sinks if j < m else j - m in rows[i]
        q = heads_of(x[st[b]:st[b + 1]], k, H, Hkv, dh)[0]
        wo, wl = aref.definition(q, kv[:, 0], kv[:, 1], mask)
        _, _, eo, el = aref.forward(q, kv[:, 0], kv[:, 1], mask, TDT[dtype])
        aref.inside(o[st[b]:st[b + 1]].reshape(k, H, dh), wo, eo, f"o[{b}]")
        aref.inside(lse[st[b]:st[b + 1]], wl, el.nan_to_num(), f"lse[{b}]")


@TYPES
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("cached,n,window,sinks,keys,value", [
    (0, 9, ALL, 0, [0], INF), (0, 9, ALL, 0, [0, 2, 5], math.nan), (300, 20, 64, 2, range(200, 312), INF), (300, 70, 80, 0, [290, 302, 330], -INF),
    (2000, 5, ALL, 0, range(2005), INF), (1500, 90, 100, 0, range(1400, 1590), INF), (100, 90, ALL, 0, [50], math.nan)])
def test_scores_that_are_not_finite_reach_the_rows_that_see_them(dtype, dh, cached, n, window, sinks, keys, value):
    """queries are negative where these keys hold `value`: inf gives scores of -inf; rows that do not see them are what they were"""
    print(f"not finite dtype={dtype} dh={dh} cached={cached} rows={n} W={window} {len(keys)} x {value}", flush=True)
    H, Hkv, page, keys = 2, 1, 16, list(keys)
    x = draw((cached + n, (H + 2 * Hkv) * dh), 31, dtype)
    x[:, :H * dh:dh] = -x[:, :H * dh:dh].abs() - 0.25
    x[keys, H * dh] = value
    c = Cache(dtype, [cached + n], Hkv, dh, page, 7)
    if cached:
        c.append(x[:cached].to(DEV), [0, cached], [0], H)
    c.append(x[cached:].to(DEV), [0, n], [cached], H)
    parents = [ref.random_parents(random.Random(3), n, "deep")]
    depth, seen = tree(parents)
    o, lse = attend(c, x[cached:].to(DEV), [0, n], [cached], depth, seen, H, n, window, sinks)
    rows = ref.seen_rows(parents[0])
    mask = mask_of(cached, rows, [len(r) - 1 for r in rows], window, sinks, cached + n)
    q, k, v = heads_of(x, cached + n, H, Hkv, dh)
    wo, wl = aref.definition(q[cached:], k, v, mask)
    plain, some = k.clone(), torch.zeros(cached + n, dtype=torch.bool)
    plain[keys, :, 0], some[keys] = 0.0, True
    _, _, eo, el = aref.forward(q[cached:], plain, v, mask & ~some, TDT[dtype])
    aref.inside(o.reshape(n, H, dh), wo, eo, "o")
    aref.inside(lse, wl, el.nan_to_num(), "lse")


@TYPES
def test_rows_of_nobody_stay_as_they_were(dtype):
    H, Hkv, dh, page = 2, 2, 64, 16
    c = Cache(dtype, [50, 50], Hkv, dh, page, 2)
    c.data.normal_()
    x = draw((47, (H + 2 * Hkv) * dh), 3, dtype)
    x[40:] = float("nan")
    parents = [ref.random_parents(random.Random(3), 20, "level")] * 2
    for n in (20, 15):                                          # rows beyond max_new as well
        depth, seen = tree(parents, max_new=n, rows=47)
        o, lse = attend(c, x.to(DEV), [0, 20, 40], [3, 0], depth, seen, H, n, ALL, 0, rows=47)
        mine = torch.tensor([r < 40 and r % 20 < n for r in range(47)])
        assert bool((o[~mine] == 77).all()) and bool((lse[~mine] == 77).all())
        assert bool(torch.isfinite(o[mine]).all()) and not bool((lse[mine] == 77).any())


@TYPES
@pytest.mark.parametrize("cached,counts,H,Hkv,dh", [([6000, 2000, 50], [1, 300, 400], 8, 1, 64), ([30000, 5, 700], [64, 40, 64], 2, 1, 32), ([4000], [7], 8, 8, 128), ([9000, 9000], [1, 2], 4, 1, 32), ([700], [200], 2, 2, 64)])
def test_the_workspace_is_as_large_as_it_is_said_to_be(dtype, cached, counts, H, Hkv, dh):
    page = 32
    c = Cache(dtype, [a + b for a, b in zip(cached, counts)], Hkv, dh, page, 3)
    c.data.normal_()
    st = starts_of(counts)
    x = draw((st[-1], (H + 2 * Hkv) * dh), 4, dtype).to(DEV)
    depth, seen = tree([ref.random_parents(random.Random(3), k, "level") for k in counts])
    want, want_lse = attend(c, x, st, cached, depth, seen, H, max(counts), ALL, 0)
    n = dp.dipaco_k_attention_tree_workspace_bytes(st[-1], len(counts), max(counts), H, Hkv, dh, page, c.per_doc)
    whole, ws = guarded_workspace(n)
    o, lse = attend(c, x, st, cached, depth, seen, H, max(counts), ALL, 0, ws=ws)
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    assert bool((whole[:4096] == 170).all()) and bool((whole[4096 + n:] == 170).all())


def test_a_chain_is_a_chunk():
    """the rows of a chain of drafts are those of dipaco_k_attention_paged, which sees each row's predecessors"""
    for dtype in (dp.F32, dp.BF16):
        for counts, cached in (([6, 3], [700, 30]), ([90, 40], [100, 1000])):
            c, x, st = filled(dtype, cached, counts, 4, 2, 64, 16, 3)
            depth, seen = tree([list(range(-1, k - 1)) for k in counts])
            o, lse = attend(c, x.to(DEV), st, cached, depth, seen, 4, max(counts), 500, 2)
            want, want_lse = c.attend(x.to(DEV), st, cached, 4, max(counts), 500, 2)
            tol = 2e-5 if dtype == dp.F32 else 3 * aref.half_step(TDT[dtype])
            assert float((o.double() - want.double()).abs().max()) <= tol * float(want.double().abs().max())
            assert float((lse - want_lse).abs().max()) <= 2e-5 * 8


def test_offsets_beyond_32_bits():
    dtype, H, Hkv, dh, page, n_pages = dp.BF16, 8, 8, 128, 64, 1 << 16
    data = torch.empty((n_pages, 2, Hkv, page, dh), dtype=torch.bfloat16, device=DEV)
    c = Cache(dtype, [200], Hkv, dh, page, 2)
    c.data, c.n_pages = data, n_pages
    c.table = [[n_pages - 1, 5, n_pages - 7, 40000]]
    c.pages = i32(c.table)
    for p in c.table[0]:
        data[p] = float("nan")
    x = draw((200, (H + 2 * Hkv) * dh), 4, dtype)
    c.append(x[:150].to(DEV), [0, 150], [0], H)
    c.append(x[150:].to(DEV), [0, 50], [150], H)
    parents = [ref.random_parents(random.Random(3), 50, "level")]
    depth, seen = tree(parents)
    o, lse = attend(c, x[150:].to(DEV), [0, 50], [150], depth, seen, H, 50, ALL, 0)
    rows = ref.seen_rows(parents[0])
    kv = c.kv[0].double()
    wo, wl, eo, el = aref.forward(heads_of(x[150:], 50, H, Hkv, dh)[0], kv[:, 0], kv[:, 1], mask_of(150, rows, [len(r) - 1 for r in rows], ALL, 0, 200), TDT[dtype])
    aref.inside(o.reshape(50, H, dh), wo, eo, "o")
    aref.inside(lse, wl, el, "lse")


# ---- the step as a whole -----------------------------------------------------------------------------------------------
class Step:
    """Drafted decoding of a batch with a stand-in for the path's layers: token t's q | k | v of layer l is a row of a table, logits are a
    product of the attention's output.  All buffers are made once, so that the step can be captured."""
    H, Hkv, dh, page, V, layers = 4, 2, 64, 16, 504, 3

    def __init__(self, dtype, B, max_new, seed=1):
        self.dtype, self.B, self.n, self.T = dtype, B, max_new, B * max_new
        g = torch.Generator(device=DEV).manual_seed(seed)
        t, width = TDT[dtype], (self.H + 2 * self.Hkv) * self.dh
        self.table = [torch.randn(self.V, width, device=DEV, generator=g).to(t) for _ in range(self.layers)]
        self.head = torch.randn(self.layers * self.H * self.dh, self.V, device=DEV, generator=g) * 0.2
        self.c = [Cache(dtype, [300] * B, self.Hkv, self.dh, self.page, 3) for _ in range(self.layers)]
        for c in self.c:
            c.data.zero_()
        self.pages = self.c[0].pages
        z = lambda *s, d=torch.int32: torch.zeros(s, dtype=d, device=DEV)
        self.tokens, self.parent, self.row_start, self.cache_len = z(self.T), z(self.T), z(B + 1), z(B)
        self.depth, self.seen = z(self.T), z(self.T, -(-max_new // 64), d=torch.int64)
        self.u, self.v = z(self.T, d=torch.float32), z(B, d=torch.float32)
        self.qkv, self.o = [z(self.T, width, d=t) for _ in range(self.layers)], [z(self.T, self.H * self.dh, d=t) for _ in range(self.layers)]
        self.target, self.out = z(self.T, self.V, d=torch.float32), z(self.T, self.layers * self.H * self.dh, d=torch.float32)
        self.path, self.kept, self.next = z(B, max_new), z(B), z(B)
        c = self.c[0]
        self.ws = torch.empty(dp.dipaco_k_attention_tree_workspace_bytes(self.T, B, max_new, self.H, self.Hkv, self.dh, self.page, c.per_doc), dtype=torch.uint8, device=DEV)
        self.vws = torch.empty(dp.dipaco_k_draft_verify_workspace_bytes(self.T, B, self.V), dtype=torch.uint8, device=DEV)

    def layer_inputs(self, l, tokens):
        """with the tokens' ids alone: a row's keys do not depend on what it saw, so that the cache's contents are known"""
        return self.table[l][tokens.long()]

    def logits(self, rows, out, target):
        dp.dipaco_k_gemm(dp.F32, False, False, False, rows, self.V, out.shape[1], out, self.head, target)

    def run(self):
        T, B, n, c = self.T, self.B, self.n, self.c[0]
        dp.dipaco_k_draft_tree(self.parent, self.row_start, self.depth, self.seen, T, B, n)
        width = self.H * self.dh
        for l in range(self.layers):
            self.qkv[l].copy_(self.layer_inputs(l, self.tokens))
            dp.dipaco_k_cache_append(self.dtype, self.qkv[l], self.row_start, self.cache_len, self.pages, self.c[l].data, T, B, self.H, self.Hkv, self.dh, c.n_pages,
                                     self.page, c.per_doc)
            dp.dipaco_k_attention_tree(self.dtype, self.qkv[l], self.row_start, self.cache_len, self.depth, self.seen, self.pages, self.c[l].data, self.o[l], None, T, B,
                                       n, self.H, self.Hkv, self.dh, c.n_pages, self.page, c.per_doc, 200, 4, self.ws)
            self.out[:, l * width:(l + 1) * width].copy_(self.o[l])
        self.logits(T, self.out, self.target)
        dp.dipaco_k_draft_verify(dp.F32, self.target, None, self.tokens, self.parent, self.row_start, self.u, self.v, self.path, self.kept, self.next, T, B, n, self.V,
                                 0.0, 1.0, False, self.vws)
        dp.dipaco_k_cache_keep(self.dtype, self.path, self.kept, self.cache_len, self.pages, [x.data for x in self.c], B, n, self.Hkv, self.dh, c.n_pages, self.page,
                               c.per_doc)
        self.cache_len += self.kept

    def one(self, caches, texts):
        """the logits behind each text, whose last token is appended to caches that hold the tokens in front of it"""
        st, lens = list(range(self.B + 1)), [len(t) - 1 for t in texts]
        out, target = [], torch.zeros((self.B, self.V), device=DEV)
        for l, c in enumerate(caches):
            x = self.layer_inputs(l, torch.tensor([t[-1] for t in texts], device=DEV))
            c.append(x, st, lens, self.H)
            out.append(c.attend(x, st, lens, self.H, 1, 200, 4)[0].float())
        self.logits(self.B, torch.cat(out, 1), target)
        return target


@TYPES
def test_drafted_decoding_writes_the_text_that_decoding_token_by_token_writes(dtype):
    """Greedy: every step's drafts hold the right continuation here and there.  The texts are those of single tokens over caches that never held
    a refused draft, and in the end so are the caches."""
    B, n, steps = 4, 12, 6
    s = Step(dtype, B, n)
    plain = [Cache(dtype, [300] * B, s.Hkv, s.dh, s.page, 9) for _ in range(s.layers)]
    for c in plain:
        c.data.zero_()
    rng = random.Random(2)
    texts = [[rng.randrange(s.V)] for _ in range(B)]                # decided token by token, ahead of the drafts
    margins = []
    while min(len(t) for t in texts) < 1 + steps * n:
        for b, x in enumerate(s.one(plain, texts)):
            top = torch.topk(x, 2).values
            margins.append(float((top[0] - top[1]) / x.abs().max()))
            texts[b].append(int(x.argmax()))
    # a greedy step is decided by scores that both ways round differently: with 16 bits of probabilities or fewer, 2^-8 and the sum's own roundings
    safe = 0.05 if dtype == dp.BF16 else 1e-4
    done = [[t[0]] for t in texts]
    for step in range(steps):
        parents, tokens, counts = [], [], []
        for b in range(B):
            k = n if (step + b) % 4 else (step + b) % 8 // 4        # now and then a document has one row, or none
            p = ref.random_parents(rng, k, rng.choice(["level", "deep", "chain"]))
            at = len(done[b]) - 1
            t, right = [], {0: 0} if k else {}
            for i in range(k):
                up = ref.parent_of(p[i], i)
                good = texts[b][at + right[up] + 1] if up in right and up >= 0 else None
                if i == 0:
                    t.append(done[b][-1])
                elif good is not None and rng.random() < 0.7:
                    t.append(good)
                    right[i] = right[up] + 1
                else:
                    t.append(rng.randrange(s.V))
                    if good is not None and t[-1] == good:
                        right[i] = right[up] + 1
            parents.append(p)
            tokens.append(t)
            counts.append(k)
        st = starts_of(counts)
        pad = [0] * (s.T - st[-1])
        s.tokens.copy_(i32([x for t in tokens for x in t] + pad))
        s.parent.copy_(i32([x for p in parents for x in p] + pad))
        s.row_start.copy_(i32(st))
        assert s.cache_len.tolist() == [len(d) - 1 for d in done]
        s.run()
        path, kept, token = s.path.tolist(), s.kept.tolist(), s.next.tolist()
        for b in range(B):
            if counts[b]:
                done[b] += [tokens[b][r] for r in path[b][1:kept[b]]] + [token[b]]
                at = len(done[b])
                wrong = [i for i in range(at) if done[b][i] != texts[b][i]]
                if wrong:                                           # only where the decision was no decision
                    i = wrong[0]
                    assert margins[(i - 1) * B + b] < safe, (step, b, i, margins[(i - 1) * B + b])
                    pytest.skip("a text hangs on a score that two roundings decide differently")
            else:
                assert kept[b] == 0 and token[b] == -1
    assert max(len(d) for d in done) > steps + 4                    # drafts did stay
    for l in range(s.layers):                                       # slots of tokens that have been decided
        for b in range(B):
            for p in range(len(done[b]) - 1):
                got = s.c[l].data[s.c[0].table[b][p // s.page], :, :, p % s.page]
                want = s.table[l][done[b][p], s.H * s.dh:].reshape(2, s.Hkv, s.dh)
                assert torch.equal(got, want), (l, b, p)


def fill(s, step):
    """rows, trees and lengths of a step, other ones for every step"""
    rng = random.Random(step)
    counts = [rng.randint(0, s.n) for _ in range(s.B)]
    counts[step % s.B] = s.n
    st = starts_of(counts)
    pad = [0] * (s.T - st[-1])
    s.parent.copy_(i32([x for k in counts for x in ref.random_parents(rng, k, "level")] + pad))
    s.tokens.copy_(i32([rng.randrange(s.V) for _ in range(st[-1])] + pad))
    s.row_start.copy_(i32(st))
    s.cache_len.copy_(i32([rng.randint(0, 250) for _ in range(s.B)]))
    g = torch.Generator().manual_seed(step)
    s.u.copy_(torch.rand(s.T, generator=g) * 0.2)
    s.v.copy_(torch.rand(s.B, generator=g))
    for l, c in enumerate(s.c):
        c.data.copy_(torch.randn(c.data.shape, generator=torch.Generator().manual_seed(100 * step + l)).to(c.data.dtype))


def outcome(s):
    return [x.clone() for x in (s.path, s.kept, s.next, s.cache_len, s.target, *s.o, *[c.data for c in s.c])]


@TYPES
def test_a_step_captured_and_replayed_beside_eager_work(dtype):
    """rows, trees, lengths and random numbers change between replays; two captured steps have workspaces of their own and run at once"""
    eager, steps = Step(dtype, 3, 14), [Step(dtype, 3, 14), Step(dtype, 3, 14)]
    side, graphs = torch.cuda.Stream(), []
    for s in steps:
        fill(s, 0)
        s.run()                                                     # library products choose what they use before the capture
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.run()
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for k in range(4):
        for s, step in zip(steps, (2 * k, 2 * k + 1)):
            fill(s, step)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for s, step in zip(steps, (2 * k, 2 * k + 1)):
            fill(eager, step)
            rows = int(eager.row_start[-1])
            eager.run()
            torch.cuda.synchronize()
            for i, (a, b) in enumerate(zip(outcome(s), outcome(eager))):
                if i >= 4 and i < 5 + s.layers:                     # rows of nobody keep what they held
                    a, b = a[:rows], b[:rows]
                assert torch.equal(a, b), (k, step, i)


def test_long_documents_captured_and_replayed_beside_eager_work():
    """lengths and trees change between replays, and with them how the call is cut"""
    dtype, H, Hkv, dh, page, B, n = dp.BF16, 4, 2, 64, 64, 3, 40
    c = Cache(dtype, [6000] * B, Hkv, dh, page, 2)
    c.data.normal_()
    T, words = B * n, 1
    x = torch.zeros((T, (H + 2 * Hkv) * dh), dtype=TDT[dtype], device=DEV)
    st, lens, depth, seen = i32([n * b for b in range(B + 1)]), i32([0] * B), i32([0] * T), torch.zeros((T, words), dtype=torch.int64, device=DEV)
    o, lse = torch.zeros((T, H * dh), dtype=TDT[dtype], device=DEV), torch.zeros((T, H), device=DEV)
    ws = torch.empty(dp.dipaco_k_attention_tree_workspace_bytes(T, B, n, H, Hkv, dh, page, c.per_doc), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        dp.dipaco_k_attention_tree(dtype, x, st, lens, depth, seen, c.pages, c.data, o, lse, T, B, n, H, Hkv, dh, c.n_pages, page, c.per_doc, ALL, 0, ws)
    for k in range(4):
        rng = random.Random(k)
        counts, at = [[40, 40, 40], [1, 40, 30], [0, 0, 5], [40, 9, 17]][k], [[5900, 10, 3000], [0, 5000, 5900], [0, 0, 4000], [200, 5900, 5800]][k]
        starts = starts_of(counts)
        d, m = tree([ref.random_parents(rng, a, "level") for a in counts], max_new=n, rows=T, starts=starts)
        x.copy_(draw((T, (H + 2 * Hkv) * dh), 90 + k, dtype))
        for to, frm in ((depth, d), (seen, m), (st, i32(starts)), (lens, i32(at))):
            to.copy_(frm)
        graph.replay()
        torch.cuda.synchronize()
        eo, el = attend(c, x, starts, at, d, m, H, n, ALL, 0, rows=T)
        torch.cuda.synchronize()
        rows = starts[-1]
        assert torch.equal(eo[:rows], o[:rows]) and torch.equal(el[:rows], lse[:rows]) and bool(torch.isfinite(el[:rows]).all())


def test_on_another_stream():
    s, t = Step(dp.BF16, 3, 9), Step(dp.BF16, 3, 9)
    fill(s, 5)
    fill(t, 5)
    torch.cuda.synchronize()
    s.run()
    other = torch.cuda.Stream()
    with torch.cuda.stream(other):
        t.run()
    torch.cuda.synchronize()
    rows = int(s.row_start[-1])
    for i, (a, b) in enumerate(zip(outcome(s), outcome(t))):
        assert torch.equal(a[:rows], b[:rows]) if 4 <= i < 5 + s.layers else torch.equal(a, b), i
