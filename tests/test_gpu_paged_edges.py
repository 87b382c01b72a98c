"""Attention over a paged cache at its edges: rows whose visible scores are infinite."""
import math

import pytest
import torch

import attention_reference as ref
import paper_2403_10616_amd as dp
from gpu_util import DEV
from test_gpu_paged import Cache, i32
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
