"""A paged cache and the attention of new tokens over it, against copies and the definition in 64 bits."""
import random

import pytest
import torch

import attention_reference as ref
import paper_2403_10616_amd as dp
from gpu_util import DEV
from test_gpu_window import ALL, TDT, draw, fwd, heads_of, within

pytestmark = pytest.mark.gpu


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


class Cache:
    """Documents of the given lengths on shuffled pages; `kv` holds their keys and values as the reference sees them"""

    def __init__(self, dtype, capacities, Hkv, dh, page, seed, spare=3):
        self.dtype, self.Hkv, self.dh, self.page = dtype, Hkv, dh, page
        used = [-(-n // page) for n in capacities]
        self.per_doc, self.n_pages = max(max(used), 1), sum(used) + spare
        order = list(range(self.n_pages))
        random.Random(seed).shuffle(order)
        self.table = [[order.pop() for _ in range(n)] + [-1] * (self.per_doc - n) for n in used]
        self.pages = i32(self.table)
        self.data = torch.full((self.n_pages, 2, Hkv, page, dh), float("nan"), dtype=TDT[dtype], device=DEV)
        self.kv = [torch.zeros((n, 2, Hkv, dh), dtype=TDT[dtype]) for n in capacities]

    def append(self, qkv, starts, lens, H):
        T, B = starts[-1], len(lens)
        dp.dipaco_k_cache_append(self.dtype, qkv, i32(starts), i32(lens), self.pages, self.data, T, B, H, self.Hkv, self.dh, self.n_pages, self.page,
                                 self.per_doc)
        x = qkv.cpu()
        for b in range(B):
            n = starts[b + 1] - starts[b]
            self.kv[b][lens[b]:lens[b] + n] = x[starts[b]:starts[b + 1], H * self.dh:].reshape(n, 2, self.Hkv, self.dh)

    def attend(self, qkv, starts, lens, H, max_new, window, sinks, rows=None, want_lse=True):
        T, B = starts[-1] if rows is None else rows, len(lens)
        o = torch.full((T, H * self.dh), 77.0, dtype=TDT[self.dtype], device=DEV)
        lse = torch.full((T, H), 77.0, device=DEV) if want_lse else None
        ws = torch.full((dp.dipaco_k_attention_paged_workspace_bytes(T, B, max_new, H, self.Hkv, self.dh, self.page, self.per_doc),), 255,
                        dtype=torch.uint8, device=DEV)
        dp.dipaco_k_attention_paged(self.dtype, qkv, i32(starts), i32(lens), self.pages, self.data, o, lse, T, B, max_new, H, self.Hkv, self.dh, self.n_pages,
                                    self.page, self.per_doc, window, sinks, ws)
        return o, lse


def starts_of(counts):
    s = [0]
    for n in counts:
        s.append(s[-1] + n)
    return s


def check(dtype, cached, new, H, Hkv, dh, page, window, sinks, seed=3, scale=1.0):
    print(f"paged dtype={dtype} cached={cached} new={new} H={H} Hkv={Hkv} dh={dh} page={page} W={window} sinks={sinks}", flush=True)
    c = Cache(dtype, [a + b for a, b in zip(cached, new)], Hkv, dh, page, seed)
    if any(cached):
        st = starts_of(cached)
        c.append(draw((st[-1], (H + 2 * Hkv) * dh), seed, dtype).to(DEV), st, [0] * len(cached), H)
    st = starts_of(new)
    x = draw((st[-1], (H + 2 * Hkv) * dh), seed + 1, dtype, scale)
    c.append(x.to(DEV), st, cached, H)
    o, lse = c.attend(x.to(DEV), st, cached, H, max(new), window, sinks)
    for b, (m, n) in enumerate(zip(cached, new)):
        if not n:
            continue
        kv = c.kv[b].double()
        q = heads_of(x[st[b]:st[b + 1]], n, H, Hkv, dh)[0]
        wo, wl, eo, el = ref.forward(q, kv[:, 0], kv[:, 1], ref.sees(m, n, m + n, window, sinks), TDT[dtype])
        within(o[st[b]:st[b + 1]].reshape(n, H, dh), wo, eo, f"o[{b}]")
        within(lse[st[b]:st[b + 1]], wl, el, f"lse[{b}]")
    o2, lse2 = c.attend(x.to(DEV), st, cached, H, max(new), window, sinks)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    o3, _ = c.attend(x.to(DEV), st, cached, H, max(new), window, sinks, want_lse=False)
    assert torch.equal(o, o3)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("cached,new,H,Hkv,dh,page", [([0], [1], 2, 2, 64, 16), ([0, 5, 200], [3, 0, 33], 4, 2, 32, 16), ([100, 7], [130, 1], 2, 1, 128, 32),
                                                      ([17, 0, 64, 3], [1, 2, 1, 0], 3, 3, 64, 64), ([1], [300], 2, 2, 32, 128), ([60, 61], [65, 66], 8, 1, 64, 256)])
def test_append_writes_its_slots_and_nothing_else(dtype, cached, new, H, Hkv, dh, page):
    print(f"append dtype={dtype} cached={cached} new={new} H={H} Hkv={Hkv} dh={dh} page={page}", flush=True)
    c = Cache(dtype, [a + b for a, b in zip(cached, new)], Hkv, dh, page, 1)
    c.data.copy_(torch.randn(c.data.shape))
    want = c.data.clone().cpu()
    st = starts_of(new)
    rows = st[-1] + 5                                           # rows behind the last document belong to nobody
    x = draw((rows, (H + 2 * Hkv) * dh), 2, dtype)
    dp.dipaco_k_cache_append(dtype, x.to(DEV), i32(st), i32(cached), c.pages, c.data, rows, len(new), H, Hkv, dh, c.n_pages, page, c.per_doc)
    for b in range(len(new)):
        for r in range(new[b]):
            p = cached[b] + r
            want[c.table[b][p // page], :, :, p % page] = x[st[b] + r, H * dh:].reshape(2, Hkv, dh)
    assert torch.equal(c.data.cpu(), want)


def test_append_drops_what_has_no_page():
    """positions behind the table, entries of -1 and beyond the pages, a negative length taken as 0"""
    dtype, H, Hkv, dh, page = dp.BF16, 2, 1, 32, 16
    data = torch.zeros((4, 2, Hkv, page, dh), dtype=torch.bfloat16, device=DEV)
    pages = i32([[0, -1], [4, 1], [2, 1 << 30]])
    new, cached = [20, 20, 4], [10, 0, -3]
    st = starts_of(new)
    x = draw((st[-1], (H + 2 * Hkv) * dh), 4, dtype)
    want = data.cpu().clone()
    dp.dipaco_k_cache_append(dtype, x.to(DEV), i32(st), i32(cached), pages, data, st[-1], 3, H, Hkv, dh, 4, page, 2)
    for b, (page_id, first, n, slot) in enumerate([(0, 0, 6, 10), (1, 16, 4, 0), (2, 0, 4, 0)]):
        want[page_id, :, :, slot:slot + n] = x[st[b] + first:st[b] + first + n, H * dh:].reshape(n, 2, Hkv, dh).permute(1, 2, 0, 3)
    assert torch.equal(data.cpu(), want)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("dh,page", [(32, 16), (64, 16), (64, 64), (128, 32), (128, 256), (64, 128)])
@pytest.mark.parametrize("cached,new,H,Hkv,window,sinks", [
    ([0], [1], 1, 1, ALL, 0), ([63, 64, 65, 0], [1, 1, 1, 1], 2, 2, ALL, 0), ([500, 3], [1, 1], 8, 2, 100, 4), ([700, 129], [1, 0], 16, 1, ALL, 0),
    ([0, 30], [70, 1], 4, 2, 20, 2), ([300, 0, 5], [40, 33, 128], 3, 1, 64, 0), ([1000], [5], 6, 2, 1, 0), ([90, 257], [17, 64], 8, 8, 50, 70)])
def test_chunks_and_tokens(dtype, dh, page, cached, new, H, Hkv, window, sinks):
    check(dtype, cached, new, H, Hkv, dh, page, window, sinks)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("cached,new,H,Hkv,dh,page,window,sinks", [
    ([9000], [1], 2, 1, 64, 64, ALL, 0), ([9000, 10], [1, 1], 4, 1, 128, 16, 5000, 100), ([6000], [40], 4, 2, 32, 32, ALL, 0),
    ([3000, 0], [200, 1], 2, 2, 64, 16, 1500, 3), ([5000, 2500, 1, 0, 777], [1] * 5, 6, 2, 64, 16, ALL, 0)])
def test_long_caches(dtype, cached, new, H, Hkv, dh, page, window, sinks):
    check(dtype, cached, new, H, Hkv, dh, page, window, sinks, seed=6)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("cached,new,H,Hkv,dh,page,window,sinks", [
    ([6000, 2000, 50], [1, 300, 400], 8, 1, 64, 64, ALL, 0), ([10, 4000, 4000, 300], [500, 1, 2, 0], 8, 4, 32, 16, ALL, 0),
    ([3000, 3000], [3, 257], 4, 4, 128, 32, 2500, 8), ([5000, 0, 900], [1, 64, 64], 2, 1, 64, 16, 4000, 0)])
def test_tokens_beside_chunks(dtype, cached, new, H, Hkv, dh, page, window, sinks):
    """documents of few packed rows and long caches in one call with long chunks: each cut into splits of its own number"""
    check(dtype, cached, new, H, Hkv, dh, page, window, sinks, seed=16)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("cached,new,H,Hkv,dh,page,window,sinks", [
    ([3000, 40], [1, 1800], 6, 3, 64, 32, ALL, 0), ([2000, 500, 0], [3, 850, 1], 10, 2, 32, 16, 1200, 5), ([700, 1500], [950, 2], 9, 9, 128, 64, ALL, 0)])
def test_rows_of_many_waves(dtype, cached, new, H, Hkv, dh, page, window, sinks):
    """more rows and heads than the chip holds waves, numbers of heads that four does not divide, documents of one split beside those of several"""
    check(dtype, cached, new, H, Hkv, dh, page, window, sinks, seed=21)


def guarded_workspace(n):
    """n bytes of 255 between two runs of 4096 bytes of 170"""
    whole = torch.full((n + 8192,), 170, dtype=torch.uint8, device=DEV)
    whole[4096:4096 + n] = 255
    return whole, whole[4096:4096 + n]


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("cached,new,H,Hkv,dh", [([6000, 2000, 50], [1, 300, 400], 8, 1, 64), ([4000], [1], 8, 8, 128), ([9000, 9000], [1, 2], 4, 1, 32), ([700], [200], 2, 2, 64)])
def test_the_workspace_is_as_large_as_it_is_said_to_be(dtype, cached, new, H, Hkv, dh):
    print(f"workspace dtype={dtype} cached={cached} new={new} H={H} Hkv={Hkv} dh={dh}", flush=True)
    page = 32
    c = Cache(dtype, [a + b for a, b in zip(cached, new)], Hkv, dh, page, 3)
    c.data.normal_()
    st = starts_of(new)
    x = draw((st[-1], (H + 2 * Hkv) * dh), 4, dtype).to(DEV)
    want, want_lse = c.attend(x, st, cached, H, max(new), ALL, 0)
    n = dp.dipaco_k_attention_paged_workspace_bytes(st[-1], len(new), max(new), H, Hkv, dh, page, c.per_doc)
    whole, ws = guarded_workspace(n)
    o, lse = torch.empty_like(want), torch.empty_like(want_lse)
    dp.dipaco_k_attention_paged(dtype, x, i32(st), i32(cached), c.pages, c.data, o, lse, st[-1], len(new), max(new), H, Hkv, dh, c.n_pages, page, c.per_doc, ALL, 0, ws)
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    assert bool((whole[:4096] == 170).all()) and bool((whole[4096 + n:] == 170).all())


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("new", [[1, 1], [50, 3]])
def test_peaked_rows(dtype, new):
    check(dtype, [400, 30], new, 4, 2, 64, 16, ALL, 0, seed=8, scale=8.0)


def test_many_documents():
    rng = random.Random(5)
    check(dp.BF16, [rng.randint(0, 90) for _ in range(150)], [rng.randint(0, 2) for _ in range(150)], 2, 1, 32, 16, 40, 2, seed=9)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 2, 70]])
def test_pages_that_are_gone_hold_no_keys(dtype, new):
    """a hole inside the visible range, a document whose pages are all gone (its rows see nothing), entries beyond the pages; what the
    table does not name is never read (it holds NaN)"""
    H, Hkv, dh, page, cached = 4, 2, 64, 16, [100, 100, 100]
    c = Cache(dtype, [a + b for a, b in zip(cached, new)], Hkv, dh, page, 2)
    st = starts_of(cached)
    c.append(draw((st[-1], (H + 2 * Hkv) * dh), 3, dtype).to(DEV), st, [0, 0, 0], H)
    st = starts_of(new)
    x = draw((st[-1], (H + 2 * Hkv) * dh), 4, dtype)
    c.append(x.to(DEV), st, cached, H)
    for b, gone in enumerate([range(2, 4), range(0, c.per_doc), [0, 5]]):
        for at in gone:
            if 0 <= c.table[b][at] < c.n_pages:
                c.data[c.table[b][at]] = float("nan")
            c.table[b][at] = [-1, c.n_pages, -(1 << 31), (1 << 31) - 1][at % 4]
    c.pages = i32(c.table)
    o, lse = c.attend(x.to(DEV), st, cached, H, max(new), ALL, 0)
    for b, (m, n) in enumerate(zip(cached, new)):
        kv = c.kv[b].double()
        held = torch.tensor([0 <= c.table[b][p // page] < c.n_pages for p in range(m + n)])
        wo, wl, eo, el = ref.forward(heads_of(x[st[b]:st[b + 1]], n, H, Hkv, dh)[0], kv[:, 0], kv[:, 1], ref.sees(m, n, m + n, ALL, 0) & held, TDT[dtype])
        if b == 1:
            assert not o[st[b]:st[b + 1]].any() and bool((lse[st[b]:st[b + 1]] == -float("inf")).all())
        else:
            within(o[st[b]:st[b + 1]].reshape(n, H, dh), wo, eo, f"o[{b}]")
            within(lse[st[b]:st[b + 1]], wl, el, f"lse[{b}]")


def test_rows_of_nobody_stay_as_they_were():
    dtype, H, Hkv, dh, page = dp.BF16, 2, 2, 64, 16
    c = Cache(dtype, [50, 50], Hkv, dh, page, 2)
    st = [0, 20, 40]
    x = draw((47, (H + 2 * Hkv) * dh), 3, dtype)
    x[40:] = float("nan")
    c.append(x[:40].to(DEV), st, [3, 0], H)
    c.kv[0][:3] = 0
    c.data[c.table[0][0], :, :, :3] = 0
    o, lse = c.attend(x.to(DEV), st, [3, 0], H, 20, ALL, 0, rows=47)
    assert bool((o[40:] == 77).all()) and bool((lse[40:] == 77).all()) and bool(torch.isfinite(o[:40]).all()) and not bool((lse[:40] == 77).any())
    o, lse = c.attend(x.to(DEV), st, [3, 0], H, 15, ALL, 0, rows=47)         # rows beyond max_new as well
    for b in range(2):
        assert bool((o[st[b] + 15:st[b + 1]] == 77).all()) and not bool((lse[st[b]:st[b] + 15] == 77).any())


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(dtype, new, dh):
    """a slot in front of the window, and the slots behind the last position, hold NaN and infinities"""
    H, Hkv, page, cached, window, sinks = 2, 1, 32, 300, 100, 4
    c = Cache(dtype, [cached + new], Hkv, dh, page, 2)
    c.append(draw((cached, (H + 2 * Hkv) * dh), 3, dtype).to(DEV), [0, cached], [0], H)
    x = draw((new, (H + 2 * Hkv) * dh), 4, dtype)
    c.append(x.to(DEV), [0, new], [cached], H)
    clean, clean_lse = c.attend(x.to(DEV), [0, new], [cached], H, new, window, sinks)
    assert bool(torch.isfinite(clean).all())                    # the slots behind the last position hold NaN all the time
    for p, value in ((150, float("nan")), (5, float("inf"))):   # seen by nobody
        c.data[c.table[0][p // page], :, :, p % page] = value
    o, lse = c.attend(x.to(DEV), [0, new], [cached], H, new, window, sinks)
    tol = 4 * ref.half_step(TDT[dtype])
    assert float((o.double() - clean.double()).abs().max()) <= tol * float(clean.double().abs().max()) + 1e-5
    assert float((lse - clean_lse).abs().max()) <= 1e-4
    at = 310 if new > 1 else 300                                # a value that only rows from `at` on see
    c.data[c.table[0][at // page], 1, :, at % page, 3] = float("inf")
    o, _ = c.attend(x.to(DEV), [0, new], [cached], H, new, window, sinks)
    o, clean = o.reshape(new, H, dh), clean.reshape(new, H, dh)
    assert bool(torch.isinf(o[at - cached:, :, 3]).all())
    o[at - cached:, :, 3] = clean[at - cached:, :, 3]
    assert float((o.double() - clean.double()).abs().max()) <= tol * float(clean.double().abs().max()) + 1e-5


def test_documents_that_share_a_prefix():
    dtype, H, Hkv, dh, page = dp.BF16, 4, 2, 64, 16
    c = Cache(dtype, [64 + 16, 64 + 16], Hkv, dh, page, 2)
    c.append(draw((64, (H + 2 * Hkv) * dh), 3, dtype).to(DEV), [0, 64, 64], [0, 0], H)
    c.table[1][:4] = c.table[0][:4]
    c.pages = i32(c.table)
    x = draw((2, (H + 2 * Hkv) * dh), 4, dtype)
    x[1] = x[0]
    c.append(x.to(DEV), [0, 1, 2], [64, 64], H)
    o, lse = c.attend(x.to(DEV), [0, 1, 2], [64, 64], H, 1, ALL, 0)
    assert torch.equal(o[0], o[1]) and torch.equal(lse[0], lse[1]) and bool(torch.isfinite(o).all())


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
def test_reading_documents_piece_by_piece_gives_the_rows_of_the_whole(dtype):
    """a padded batch in one call, and the same documents chunk by chunk and then token by token over the cache, pages handed back as the
    window leaves them behind"""
    lengths, H, Hkv, dh, page, window, sinks = [150, 0, 97, 33], 4, 2, 64, 16, 40, 3
    B, S = len(lengths), max(lengths)
    x = draw((B * S, (H + 2 * Hkv) * dh), 71, dtype)
    whole, whole_lse = fwd(dtype, x.to(DEV), i32(lengths), B, S, H, Hkv, dh, window, sinks)
    c = Cache(dtype, [max(n, 1) for n in lengths], Hkv, dh, page, 4)
    done, step = [0] * B, 0
    sizes = [[70, 5, 1, 20], [3, 2, 33, 0], [0, 1, 60, 12], [64, 1, 1, 1]]
    while done != lengths:
        want = sizes[step] if step < len(sizes) else [1] * B
        new = [min(w, n - d) for w, n, d in zip(want, lengths, done)]
        step += 1
        if not any(new):
            continue
        st = starts_of(new)
        rows = torch.cat([x[b * S + d:b * S + d + n] for b, (d, n) in enumerate(zip(done, new))]).to(DEV)
        c.append(rows, st, done, H)
        o, lse = c.attend(rows, st, done, H, max(new), window, sinks)
        for b, (d, n) in enumerate(zip(done, new)):
            at = slice(b * S + d, b * S + d + n)
            tol = (2e-5 if dtype == dp.F32 else 3 * ref.half_step(TDT[dtype]))
            assert float((o[st[b]:st[b + 1]].double() - whole[at].double()).abs().max()) <= tol * float(whole[at].double().abs().max()) if n else True
            assert float((lse[st[b]:st[b + 1]].T - whole_lse[b, :, d:d + n]).abs().max()) <= 2e-5 * 8 if n else True
        done = [d + n for d, n in zip(done, new)]
        for b, d in enumerate(done):                            # pages between the sinks and the next row's window
            for p in range(-(-sinks // page), max(0, d - window + 1) // page):
                if c.table[b][p] >= 0:
                    c.data[c.table[b][p]] = float("nan")
                    c.table[b][p] = -1
        c.pages = i32(c.table)


def test_captured_and_replayed_beside_eager_work():
    """a decoding step as a graph: lengths, pages and rows change between replays"""
    dtype, H, Hkv, dh, page, B = dp.BF16, 4, 2, 64, 16, 3
    c = Cache(dtype, [400] * B, Hkv, dh, page, 2)
    st0 = [0, 300, 600, 900]
    c.append(draw((900, (H + 2 * Hkv) * dh), 3, dtype).to(DEV), st0, [0] * B, H)
    x, st, lens = torch.zeros((B, (H + 2 * Hkv) * dh), dtype=TDT[dtype], device=DEV), i32([0, 1, 2, 3]), i32([0] * B)
    o, lse = torch.empty((B, H * dh), dtype=TDT[dtype], device=DEV), torch.empty((B, H), device=DEV)
    ws = torch.empty(dp.dipaco_k_attention_paged_workspace_bytes(B, B, 1, H, Hkv, dh, page, c.per_doc), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        dp.dipaco_k_cache_append(dtype, x, st, lens, c.pages, c.data, B, B, H, Hkv, dh, c.n_pages, page, c.per_doc)
        dp.dipaco_k_attention_paged(dtype, x, st, lens, c.pages, c.data, o, lse, B, B, 1, H, Hkv, dh, c.n_pages, page, c.per_doc, 200, 4, ws)
    for k in range(4):
        rows, at = draw((B, (H + 2 * Hkv) * dh), 80 + k, dtype).to(DEV), [300 + k, 10 * k, 290 - k]
        x.copy_(rows)
        lens.copy_(torch.tensor(at, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eo, el = c.attend(rows, [0, 1, 2, 3], at, H, 1, 200, 4)
        torch.cuda.synchronize()
        assert torch.equal(eo, o) and torch.equal(el, lse)


def test_offsets_beyond_32_bits():
    """pages whose elements lie beyond 2^32 in the cache: 2^16 pages of 2 x 8 heads x 64 x 128 bf16 = 8.6e9 elements, of which five are used"""
    dtype, H, Hkv, dh, page = dp.BF16, 8, 8, 128, 64
    n_pages = 1 << 16
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
    o, lse = c.attend(x[150:].to(DEV), [0, 50], [150], H, 50, ALL, 0)
    kv = c.kv[0].double()
    wo, wl, eo, el = ref.forward(heads_of(x[150:], 50, H, Hkv, dh)[0], kv[:, 0], kv[:, 1], ref.sees(150, 50, 200, ALL, 0), TDT[dtype])
    within(o.reshape(50, H, dh), wo, eo, "o")
    within(lse, wl, el, "lse")
