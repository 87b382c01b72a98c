"""Attention over a paged cache at its edges: rows whose visible scores are infinite, documents that have outgrown their table."""
import math

import pytest
import torch

import attention_reference as ref
import paper_2403_10616_amd as dp
from gpu_util import DEV
from test_gpu_paged import Cache, i32, starts_of
from test_gpu_window import ALL, TDT, draw, fwd, heads_of

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
INF = math.inf


def rows_over_infinite_keys(dtype, cached, new, H, Hkv, dh, page, window, sinks, keys, value, gone=()):
    """One document whose queries are negative where the keys at positions `keys` hold `value` (inf: their scores are -inf; -inf: inf; nan),
    beside one of ordinary values, over the cache and, if no page is gone, in one windowed call."""
    print(f"infinite keys dtype={dtype} cached={cached} new={new} H={H} Hkv={Hkv} dh={dh} W={window} sinks={sinks} {len(keys)} x {value} gone={gone}", flush=True)
    n = cached + new
    x = draw((n, (H + 2 * Hkv) * dh), 31, dtype)
    x[:, :H * dh:dh] = -x[:, :H * dh:dh].abs() - 0.25
    for h in range(Hkv):
        x[keys, (H + h) * dh] = value
    c = Cache(dtype, [n, 40], Hkv, dh, page, 7)
    other = draw((40, (H + 2 * Hkv) * dh), 32, dtype)
    if cached:
        c.append(x[:cached].to(DEV), [0, cached, cached], [0, 0], H)
    rows, st = torch.cat([x[cached:], other]).to(DEV), [0, new, new + 40]
    c.append(rows, st, [cached, 0], H)
    held = torch.ones(n, dtype=torch.bool)
    for p in gone:
        c.table[0][p] = -1
        held[p * page:(p + 1) * page] = False
    c.pages = i32(c.table)
    o, lse = c.attend(rows, st, [cached, 0], H, max(new, 40), window, sinks)
    q, k, v = heads_of(x, n, H, Hkv, dh)
    mask = ref.sees(cached, new, n, window, sinks) & held
    wo, wl = ref.definition(q[cached:], k, v, mask)
    plain_k, some = k.clone(), torch.zeros(n, dtype=torch.bool)
    plain_k[keys, :, 0], some[keys] = 0.0, True
    _, _, eo, el = ref.forward(q[cached:], plain_k, v, mask & ~some, TDT[dtype])
    ref.inside(o[:new].reshape(new, H, dh), wo, eo, "o")
    ref.inside(lse[:new], wl, el, "lse")
    q, k, v = heads_of(other, 40, H, Hkv, dh)
    wo2, wl2, eo, el = ref.forward(q, k, v, ref.sees(0, 40, 40, window, sinks), TDT[dtype])
    ref.inside(o[new:].reshape(40, H, dh), wo2, eo, "o of the other")
    ref.inside(lse[new:], wl2, el, "lse of the other")
    if not gone:
        ow, lw = fwd(dtype, x.to(DEV), None, 1, n, H, Hkv, dh, window, sinks)
        assert torch.equal(torch.isnan(ow[cached:]).cpu(), torch.isnan(wo.reshape(new, -1)))
        assert torch.equal((lw[0, :, cached:].T == -INF).cpu(), wl == -INF)
    return wo, wl


@TYPES
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("cached,new,H,Hkv,window,sinks,keys,gone", [
    (0, 1, 2, 1, ALL, 0, [0], ()), (0, 5, 2, 2, ALL, 0, [0], ()), (0, 90, 4, 1, 1, 0, [0, 7, 40, 89], ()), (300, 3, 2, 1, 64, 2, range(200, 303), ()),
    (2000, 1, 2, 1, ALL, 0, range(2001), ()), (2000, 1, 2, 1, ALL, 0, [p for p in range(2001) if p != 700], ()), (1500, 120, 2, 2, ALL, 0, range(1540), ()),
    (1500, 2, 4, 4, 1000, 3, range(1502), ()), (2500, 70, 2, 1, ALL, 5, [p for p in range(2570) if p not in (3, 2000)], ()),
    (64, 40, 2, 1, ALL, 0, range(60, 90), range(0, 3)), (64, 40, 2, 1, 8, 0, range(64, 104), range(4, 7)), (64, 2, 2, 1, ALL, 0, range(66), range(0, 5)),
    (2000, 1, 2, 1, ALL, 0, range(0, 2001), range(0, 100))])
def test_a_row_whose_visible_scores_are_all_minus_infinity_is_not_a_row_that_sees_nothing(dtype, dh, cached, new, H, Hkv, window, sinks, keys, gone):
    wo, wl = rows_over_infinite_keys(dtype, cached, new, H, Hkv, dh, 16, window, sinks, list(keys), INF, list(gone))
    if len(keys) == 1 or len(keys) == cached + new and len(gone) < 5:
        assert bool(torch.isnan(wo[0]).all()) and bool((wl[0] == -INF).all())      # the cases are what they are meant to be


@TYPES
@pytest.mark.parametrize("value", [-INF, math.nan])
@pytest.mark.parametrize("cached,new,window,keys", [(0, 1, ALL, [0]), (0, 70, 1, [0, 69]), (2000, 1, ALL, [1234]), (1500, 90, 40, [1490, 1530]), (2000, 1, ALL, range(2001))])
def test_a_score_that_is_infinite_or_no_number_reaches_the_rows_that_see_it(dtype, value, cached, new, window, keys):
    rows_over_infinite_keys(dtype, cached, new, 2, 1, 64, 16, window, 0, list(keys), value)


@TYPES
@pytest.mark.parametrize("dh,page", [(32, 16), (64, 32), (128, 16)])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (4, 1)])
@pytest.mark.parametrize("cached,new,window,sinks", [
    ([70, 64, 60], [1, 1, 1], 20, 0), ([70, 64, 60], [3, 30, 30], 20, 2), ([70, 64, 3], [1, 60, 90], 20, 0), ([90, 0, 64], [40, 5, 1], ALL, 0),
    ([1 << 30, (1 << 28) + 7, 1000], [2, 33, 1], ALL, 0), ([(1 << 30) - 5, 1 << 29, 100], [9, 1, 40], (1 << 31) - 1, 0), ([1 << 30, 84, 83], [1, 1, 1], 20, 5)])
def test_rows_of_a_document_that_has_outgrown_its_table(dtype, dh, page, H, Hkv, cached, new, window, sinks):
    """64 positions a table: rows keep their positions, and see of the table what a row at such a position sees"""
    print(f"outgrown dtype={dtype} cached={cached} new={new} H={H} Hkv={Hkv} dh={dh} page={page} W={window} sinks={sinks}", flush=True)
    t, room, B = TDT[dtype], 64, len(cached)
    c = Cache(dtype, [room] * B, Hkv, dh, page, 3)
    data = draw(tuple(c.data.shape), 5, dtype)
    c.data.copy_(data)
    st = starts_of(new)
    x = draw((st[-1], (H + 2 * Hkv) * dh), 6, dtype)
    rows = x.to(DEV)
    dp.dipaco_k_cache_append(dtype, rows, i32(st), i32(cached), c.pages, c.data, st[-1], B, H, Hkv, dh, c.n_pages, page, c.per_doc)
    for b, (m, n) in enumerate(zip(cached, new)):
        for p in range(m, min(m + n, room)):
            data[c.table[b][p // page], :, :, p % page] = x[st[b] + p - m, H * dh:].reshape(2, Hkv, dh)
    assert torch.equal(c.data.cpu(), data)
    o, lse = c.attend(rows, st, cached, H, max(new), window, sinks)
    for b, (m, n) in enumerate(zip(cached, new)):
        kv = torch.cat([data[p] for p in c.table[b]], 2).double().permute(2, 0, 1, 3)           # [position, 2, Hkv, dh]
        mask = ref.sees(m, n, room, window, sinks)
        q = heads_of(x[st[b]:st[b + 1]], n, H, Hkv, dh)[0]
        wo, wl = ref.definition(q, kv[:, 0], kv[:, 1], mask)
        _, _, eo, el = ref.forward(q, kv[:, 0], kv[:, 1], mask, t)
        ref.inside(o[st[b]:st[b + 1]].reshape(n, H, dh), wo, eo, f"o[{b}]")
        ref.inside(lse[st[b]:st[b + 1]], wl, el.nan_to_num(), f"lse[{b}]")
