"""A step of drafted decoding against its statement on the host: trees, which drafts stay, moving what stays, and the step as a whole."""
import math
import random

import pytest
import torch

import draft_reference as ref
import paper_2403_10616_amd as dp
from gpu_util import DEV
from test_gpu_paged import Cache, guarded_workspace, i32, starts_of
from test_gpu_window import ALL, TDT, draw

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])


# ---- trees -----------------------------------------------------------------------------------------------------------
def tree(parents, max_new=None, rows=None, starts=None):
    """depth and seen of a batch of trees, on the device; what is not written holds 77"""
    st = starts_of([len(p) for p in parents]) if starts is None else starts
    T, n = st[-1] if rows is None else rows, max(len(p) for p in parents) if max_new is None else max_new
    given = i32([x for p in parents for x in p] + [0] * (T - sum(len(p) for p in parents)))
    depth = torch.full((T,), 77, dtype=torch.int32, device=DEV)
    seen = torch.full((T, -(-n // 64)), 77, dtype=torch.int64, device=DEV)
    dp.dipaco_k_draft_tree(given, i32(st), depth, seen, T, len(parents), n)
    return depth, seen


@pytest.mark.parametrize("shape", ["chain", "star", "level", "deep", "forest"])
@pytest.mark.parametrize("counts", [[1], [16], [63, 0, 64, 65], [5] * 70, [128, 129, 1, 300], [1024, 3, 700]])
def test_trees(shape, counts):
    print(f"trees {shape} {counts}", flush=True)
    rng = random.Random(3)
    parents = [ref.random_parents(rng, n, shape) for n in counts]
    depth, seen = tree(parents)
    rows = [r for p in parents for r in ref.seen_rows(p)]
    assert depth.tolist() == [len(r) - 1 for r in rows]
    words = -(-max(counts) // 64)
    assert seen.tolist() == [ref.words_of(r, words) for r in rows]


def test_tree_rows_of_nobody_stay_as_they_were():
    parents = [[-1, 0, 1, 1, 2], [-1, 0, 0]]
    depth, seen = tree(parents, max_new=3, rows=11)
    assert depth.tolist() == [0, 1, 2, 77, 77, 0, 1, 1, 77, 77, 77]
    assert seen[:, 0].tolist() == [1, 3, 7, 77, 77, 1, 3, 5, 77, 77, 77]
    depth, _ = tree(parents, max_new=5, rows=8, starts=[-4, 5, 100])          # bounds outside the call are taken as the nearest inside
    assert depth.tolist() == [0, 1, 2, 2, 3, 0, 1, 1]


# ---- which drafts stay ------------------------------------------------------------------------------------------------
def verify(dtype, target, draft, tokens, parents, u, v, temperature=1.0, draft_temperature=1.0, distinct=False, max_new=None, starts=None, stream=None, ws=None):
    st = starts_of([len(p) for p in parents]) if starts is None else starts
    T, B, V, n = target.shape[0], len(parents), target.shape[1], max(len(p) for p in parents) if max_new is None else max_new
    dev = [x if x is None else x.to(DEV) for x in (target, draft)]
    path = torch.full((B, n), 77, dtype=torch.int32, device=DEV)
    kept, token = (torch.full((B,), 77, dtype=torch.int32, device=DEV) for _ in range(2))
    if ws is None:
        ws = torch.full((dp.dipaco_k_draft_verify_workspace_bytes(T, B, V),), 255, dtype=torch.uint8, device=DEV)
    given = [x for p in parents for x in p]
    dp.dipaco_k_draft_verify(dtype, *dev, i32(tokens), i32(given + [0] * (T - len(given))), i32(st), u.to(DEV), v.to(DEV), path, kept, token, T, B, n, V,
                             temperature, draft_temperature, distinct, ws, stream=stream)
    return path.tolist(), kept.tolist(), token.tolist()


def drafts(rng, g, draft, parents, mode, temperature):
    """tokens that a draft proposes: drawn, drawn without replacement, or picked; a few at random, a few that are no token"""
    V, out = draft.shape[1], [0] * len(parents)
    used = {}
    for i, given in enumerate(parents):
        p = ref.parent_of(given, i)
        q = ref.distribution(draft[max(p, 0)], temperature)
        before = used.setdefault(p, [])
        if mode == "picked":
            out[i] = int(torch.topk(q, min(V, len(before) + 1)).indices[-1])
        else:
            w = q.clone()
            if mode == "distinct" and len(before) < V:
                w[before] = 0.0
            if float(w.sum()) == 0:
                w = q
            out[i] = int(torch.multinomial(w, 1, generator=g))
        if rng.random() < 0.04:
            out[i] = rng.choice([-1, V, 1 << 30, rng.randrange(V)])
        if 0 <= out[i] < V:
            before.append(out[i])
    return out


def check_verify(dtype, counts, shape, V, mode, temperature, draft_temperature=1.0, near=0.7, seed=1, special=None):
    print(f"verify dtype={dtype} {counts} {shape} V={V} {mode} t={temperature} {draft_temperature}", flush=True)
    rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
    st = starts_of(counts)
    T, B = st[-1], len(counts)
    draft = 2.5 * torch.randn(T, V, generator=g)
    target = (draft / draft_temperature * (temperature or 1.0) + near * torch.randn(T, V, generator=g)).to(TDT[dtype])
    draft = draft.to(TDT[dtype])
    if special:
        special(target, draft)
    parents = [ref.random_parents(rng, n, shape) for n in counts]
    tokens = [x for b in range(B) for x in drafts(rng, g, draft[st[b]:st[b + 1]], parents[b], mode, draft_temperature)]
    u, v = torch.rand(T, generator=g), torch.rand(B, generator=g)
    if B > 2:
        v[0], v[1] = 0.0, 1 - 2.0 ** -24
    given = None if mode == "picked" else draft
    path, kept, token = verify(dtype, target, given, tokens, parents, u, v, temperature, draft_temperature, mode == "distinct")
    lengths = []
    for b in range(B):
        at = slice(st[b], st[b + 1])
        want, last = ([], -1) if counts[b] == 0 else ref.walk(target[at], None if given is None else given[at], tokens[at], parents[b], u[at], v[b], temperature,
                                                               draft_temperature, mode == "distinct")
        assert path[b] == want + [-1] * (max(counts) - len(want)), (b, path[b], want)
        assert kept[b] == len(want) and token[b] == last, (b, kept[b], len(want), token[b], last)
        lengths.append(len(want))
    again = verify(dtype, target, given, tokens, parents, u, v, temperature, draft_temperature, mode == "distinct")
    assert again == (path, kept, token)
    return lengths


MODES = pytest.mark.parametrize("mode", ["drawn", "distinct", "picked"])


@TYPES
@MODES
@pytest.mark.parametrize("V", [1, 2, 7, 63, 1000, 1001, 4097])
@pytest.mark.parametrize("shape,temperature", [("chain", 1.0), ("level", 0.7), ("forest", 1.3), ("deep", 0.0)])
def test_walks(dtype, mode, V, shape, temperature):
    lengths = check_verify(dtype, [6, 0, 1, 40, 13, 25, 30, 2], shape, V, mode, temperature)
    if V >= 63 and shape == "chain" and mode != "picked":
        assert max(lengths) > 2                              # drafts do stay


@TYPES
@MODES
def test_a_vocabulary_of_many_parts(dtype, mode):
    check_verify(dtype, [6, 3, 17, 30], "level", 32000, mode, 0.9)
    check_verify(dtype, [9, 4], "deep", 50001, mode, 1.0, seed=4)


@TYPES
@MODES
@pytest.mark.parametrize("counts,shape,V,temperature", [
    ([8, 0, 5, 8] * 10, "chain", 20000, 1.0), ([16, 3, 0, 16] * 8, "level", 20011, 0.7), ([7, 16] * 16, "forest", 17001, 0.0), ([40, 0, 33] * 9, "level", 20011, 0.8),
    ([64, 50] * 6, "deep", 30001, 0.0)])
def test_sums_formed_ahead_and_in_the_walk(dtype, mode, counts, shape, V, temperature):
    """more parts of rows than all are formed of ahead of the walks: of rows with children (documents of few rows), of none (of many); documents without
    rows among them, walks that end at leaves"""
    lengths = check_verify(dtype, counts, shape, V, mode, temperature, near=0.3, seed=11)
    assert max(lengths) > 1


@MODES
def test_many_siblings(mode):
    """a row with more siblings than a wave has lanes, most of them refused; one with as many rows as a document may have"""
    check_verify(dp.F32, [100, 130, 70], "star", 300, mode, 1.0, near=4.0, seed=5)
    check_verify(dp.BF16, [1024, 40], "star", 50, mode, 1.0, near=4.0, seed=6)


@MODES
def test_other_temperatures_of_the_draft(mode):
    check_verify(dp.F32, [12, 20, 7], "level", 500, mode, 0.8, draft_temperature=0.3, seed=7)
    check_verify(dp.BF16, [12, 20, 7], "level", 500, mode, 1e-3, draft_temperature=2.0, seed=8)


@TYPES
@MODES
def test_scores_that_are_masked(dtype, mode):
    """-inf and the type's lowest value; a row of which one score is left; the draft masks other tokens than the target"""
    low = torch.finfo(TDT[dtype]).min

    def special(target, draft):
        target[:, ::3] = -math.inf
        target[:, 1::5] = low
        draft[:, ::4] = -math.inf
        target[4] = -math.inf
        target[4, 17] = -3.0
        draft[5] = low
        draft[5, 2] = 0.0

    check_verify(dtype, [20, 30, 11], "level", 120, mode, 1.0, special=special, seed=9)


@TYPES
@MODES
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_rows_that_are_no_distribution(dtype, mode, value):
    """a target row ends the walk without a token; a draft row's children are not taken"""
    def bad_target(target, draft):
        target[0, -1 if value != -math.inf else slice(None)] = value
        target[9] = value

    def bad_draft(target, draft):
        draft[1:, 3 if value != -math.inf else slice(None)] = value

    for t in (1.0, 0.0):
        assert check_verify(dtype, [6, 20, 30], "chain", 90, mode, t, special=bad_target, near=0.2, seed=10)[0] == 1
    if mode != "picked":
        check_verify_without_drafts_of_bad_rows(dtype, mode, bad_draft)


def check_verify_without_drafts_of_bad_rows(dtype, mode, special):
    g = torch.Generator().manual_seed(3)
    target = torch.randn(8, 90, generator=g).to(TDT[dtype])
    draft = target.clone()
    special(target, draft)
    tokens, parents, u, v = [5] * 8, [list(range(-1, 7))], torch.zeros(8), torch.tensor([0.37])
    path, kept, token = verify(dtype, target, draft, tokens, parents, u, v, distinct=mode == "distinct")
    want, last = ref.walk(target, draft, tokens, parents[0], u, v[0], 1.0, 1.0, mode == "distinct")
    assert len(want) == 2 and path[0] == want + [-1] * 6 and kept == [2] and token == [last]


def test_equal_scores_take_every_draft_and_the_lowest_of_equals():
    V, n = 40, 12
    s = torch.zeros(n, V)
    u = torch.full((n,), 1 - 2.0 ** -24)
    path, kept, token = verify(dp.F32, s, s, [7] * n, [list(range(-1, n - 1))], u, torch.zeros(1), distinct=True)
    assert kept == [n] and path[0] == list(range(n)) and token == [0]
    path, kept, token = verify(dp.F32, s, None, [7] * n, [list(range(-1, n - 1))], u, torch.zeros(1), temperature=0.0)
    assert kept == [1] and token == [0]
    path, kept, token = verify(dp.F32, s, None, [0] * n, [list(range(-1, n - 1))], u, torch.zeros(1), temperature=0.0)
    assert kept == [n] and token == [0]


def test_a_document_has_no_more_rows_than_are_looked_at():
    """rows beyond max_new do not exist; documents' bounds outside the call are taken as the nearest inside"""
    V, s = 30, torch.zeros(10, 30)
    path, kept, token = verify(dp.BF16, s.bfloat16(), s.bfloat16(), [3] * 10, [list(range(-1, 9))], torch.zeros(10), torch.tensor([0.5]), max_new=4)
    assert path == [[0, 1, 2, 3]] and kept == [4] and token == [15]
    path, kept, token = verify(dp.BF16, s.bfloat16(), s.bfloat16(), [3] * 10, [list(range(-1, 9)), []], torch.zeros(10), torch.tensor([0.5, 0.5]),
                               starts=[-5, 10, 12])
    assert kept == [10, 0] and token == [15, -1] and path[1] == [-1] * 10


def test_random_numbers_outside_their_range_end():
    """nothing is said of the result but that it is one of the vocabulary"""
    g = torch.Generator().manual_seed(2)
    s = torch.randn(24, 200, generator=g)
    for bad in (math.nan, -1.0, 1.0, 5.0, math.inf):
        for draft in (None, s + 1e-3 * torch.randn(24, 200, generator=g)):
            _, kept, token = verify(dp.F32, s, draft, list(range(24)), [ref.random_parents(random.Random(1), 24, "level")], torch.full((24,), bad),
                                    torch.full((1,), bad), distinct=draft is not None)
            assert 1 <= kept[0] <= 24 and 0 <= token[0] < 200


def test_offsets_of_logits_beyond_32_bits():
    """9000 rows of 2^18 scores: 2.4e9 elements; the last document's rows lie behind 2^31"""
    T, V = 9000, 1 << 18
    target = torch.zeros((T, V), dtype=torch.bfloat16, device=DEV)
    target[-6:, 1234] = 30.0
    target[-1, 1234] = 0.0
    target[-1, 200000] = 30.0
    parents = [list(range(-1, n - 1)) for n in [1000] * 8 + [994, 6]]
    path, kept, token = verify(dp.BF16, target, None, [1234] * T, parents, torch.full((T,), 0.5), torch.full((10,), 0.5))
    assert kept[:9] == [1] * 9 and kept[9] == 6 and token[9] == 200000


@TYPES
def test_verify_workspace_is_as_large_as_it_is_said_to_be(dtype):
    g = torch.Generator().manual_seed(2)
    s, d = (3 * torch.randn(30, 777, generator=g).to(TDT[dtype]) for _ in range(2))
    parents = [ref.random_parents(random.Random(b), 10, "level") for b in range(3)]
    args = (dtype, s, d, torch.randint(0, 777, (30,), generator=g).tolist(), parents, torch.rand(30, generator=g), torch.rand(3, generator=g))
    want = verify(*args)
    n = dp.dipaco_k_draft_verify_workspace_bytes(30, 3, 777)
    whole, ws = guarded_workspace(n)
    assert verify(*args, ws=ws) == want
    assert bool((whole[:4096] == 170).all()) and bool((whole[4096 + n:] == 170).all())


# ---- moving what stays ------------------------------------------------------------------------------------------------
@TYPES
@pytest.mark.parametrize("dh,page,Hkv,layers", [(32, 16, 3, 1), (64, 16, 14, 12), (128, 64, 8, 3), (64, 256, 1, 70), (128, 32, 5, 2)])
@pytest.mark.parametrize("cached,max_new", [([0, 100, 37], 16), ([5] * 9, 1), ([60, 0, 250, 15], 200)])
def test_kept_rows_move_to_their_places(dtype, dh, page, Hkv, layers, cached, max_new):
    print(f"keep dtype={dtype} dh={dh} page={page} Hkv={Hkv} layers={layers} cached={cached} max_new={max_new}", flush=True)
    rng, B = random.Random(max_new + dh), len(cached)
    c = Cache(dtype, [n + max_new for n in cached], Hkv, dh, page, 3)
    g = torch.Generator(device=DEV).manual_seed(1)
    caches = [torch.randn(c.data.shape, device=DEV, generator=g).to(TDT[dtype]) for _ in range(layers)]
    paths = []
    for b in range(B):
        kept = [max_new, 1, 0][b] if b < 3 and max_new > 1 and rng.random() < 0.5 else rng.randint(0, max_new)
        paths.append([0] * min(1, kept) + sorted(rng.sample(range(1, max_new), kept - 1)) if kept else [])
    want = [x.clone() for x in caches]
    for b, path in enumerate(paths):
        for i, r in enumerate(path):
            to, frm = cached[b] + i, cached[b] + r
            for w, old in zip(want, caches):
                w[c.table[b][to // page], :, :, to % page] = old[c.table[b][frm // page], :, :, frm % page]
    dp.dipaco_k_cache_keep(dtype, i32([p + [-1] * (max_new - len(p)) for p in paths]), i32([len(p) for p in paths]), i32(cached), c.pages, caches, B, max_new,
                           Hkv, dh, c.n_pages, page, c.per_doc)
    for got, w in zip(caches, want):
        assert torch.equal(got, w)


def test_keep_ends_where_a_path_is_none_and_leaves_rows_without_pages():
    dtype, Hkv, dh, page, n = dp.BF16, 2, 64, 16, 40
    c = Cache(dtype, [60] * 7, Hkv, dh, page, 3)
    before = torch.randn(c.data.shape, device=DEV).to(torch.bfloat16)
    cached = [10, 10, 10, 10, 10, -5, (1 << 31) - 1]
    paths = [[0, 3, 2, 9], [0, 5, 5, 9], [2, 4, 40, 41], [-1, 3, 4, 5], [1, 20, 39, -1], [0, 3, 5, 9], [0, 3, 5, 9]]
    kept = [4, 4, 4, 4, 400, 4, 4]
    done = [[(1, 3)], [(1, 5)], [(0, 2), (1, 4)], [], [(0, 1), (2, 39)], [(1, 3), (2, 5), (3, 9)], []]
    c.table[4][1] = -1                                          # positions 16 .. 31 of document 4: row 1 comes from position 30
    c.pages = i32(c.table)
    want, got = before.clone(), before.clone()
    for b, moves in enumerate(done):
        for i, r in moves:
            to, frm = max(cached[b], 0) + i, max(cached[b], 0) + r
            want[c.table[b][to // page], :, :, to % page] = before[c.table[b][frm // page], :, :, frm % page]
    dp.dipaco_k_cache_keep(dtype, i32([p + [-1] * (n - 4) for p in paths]), i32(kept), i32(cached), c.pages, [got], 7, n, Hkv, dh, c.n_pages, page, c.per_doc)
    assert torch.equal(got, want)


def test_keep_beyond_32_bit_offsets():
    dtype, Hkv, dh, page, n_pages = dp.BF16, 8, 128, 64, 1 << 16
    data = torch.zeros((n_pages, 2, Hkv, page, dh), dtype=torch.bfloat16, device=DEV)
    pages = i32([[n_pages - 1, n_pages - 5]])
    data[n_pages - 5, :, :, 6] = 3.0
    dp.dipaco_k_cache_keep(dtype, i32([[0, 10, 11]]), i32([2]), i32([60]), pages, [data], 1, 3, Hkv, dh, n_pages, page, 2)
    assert not data[n_pages - 1].any()                          # 10 is no row of a call of three
    dp.dipaco_k_cache_keep(dtype, i32([[0, 10] + [-1] * 9]), i32([2]), i32([60]), pages, [data], 1, 11, Hkv, dh, n_pages, page, 2)
    assert bool((data[n_pages - 1, :, :, 61] == 3).all()) and float(data[n_pages - 1].float().sum()) == 3 * 2 * Hkv * dh
