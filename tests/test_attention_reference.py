"""The reference of the window and paged attention tests against automatic differentiation and against differences (CPU)."""
import math

import pytest
import torch

import attention_reference as ref


def _dense(x, H, Hkv, dh, mask):
    n, G = x.shape[0], H // Hkv
    q, k, v = x[:, :H * dh].reshape(n, H, dh), x[:, H * dh:(H + Hkv) * dh].reshape(n, Hkv, dh), x[:, (H + Hkv) * dh:].reshape(n, Hkv, dh)
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(dh)
    return torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(~mask, -math.inf), 2), v)


@pytest.mark.parametrize("n,H,Hkv,dh,window,sinks", [(1, 1, 1, 4, 1, 0), (9, 2, 2, 4, 3, 0), (9, 4, 2, 4, 3, 2), (7, 3, 1, 6, 100, 0), (8, 2, 1, 4, 1, 1),
                                                     (6, 1, 1, 4, 2, 50)])
def test_reference_is_what_automatic_differentiation_gives(n, H, Hkv, dh, window, sinks):
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, (H + 2 * Hkv) * dh, generator=g, dtype=torch.float64, requires_grad=True)
    d_o = torch.randn(n, H, dh, generator=g, dtype=torch.float64)
    mask = ref.sees(0, n, n, window, sinks)
    for i in range(n):                                       # the rule, a pair at a time
        for j in range(n):
            assert bool(mask[i, j]) == (j <= i and (i - j < window or j < sinks))
    want = _dense(x, H, Hkv, dh, mask)
    (want * d_o).sum().backward()
    with torch.no_grad():
        q, k, v = (p.reshape(n, -1, dh) for p in (x[:, :H * dh], x[:, H * dh:(H + Hkv) * dh], x[:, (H + Hkv) * dh:]))
        o, lse, _, _ = ref.forward(q, k, v, mask, torch.float32)
        torch.testing.assert_close(o, want, rtol=1e-12, atol=1e-12)
        grads = ref.backward(q, k, v, o, d_o, lse, mask, torch.float32)[:3]
        got = torch.cat([t.reshape(n, -1) for t in grads], 1)
        torch.testing.assert_close(got, x.grad, rtol=1e-11, atol=1e-12)
        for at in [(0, 0), (n // 2, H * dh), (n - 1, (H + Hkv) * dh)]:       # differences
            step = torch.zeros_like(x)
            step[at] = 1e-5
            slope = ((_dense(x + step, H, Hkv, dh, mask) - _dense(x - step, H, Hkv, dh, mask)) * d_o).sum() / 2e-5
            assert abs(float(slope - got[at])) <= 1e-8


@pytest.mark.parametrize("got,want,fine", [(1.0, 1.0, True), (1.0 + 1e-3, 1.0, True), (1.1, 1.0, False), (math.nan, 1.0, False), (math.inf, 1.0, False), (1.0, math.nan, False),
                                           (1.0, math.inf, False), (math.inf, math.inf, True), (-math.inf, math.inf, False), (math.nan, math.nan, True), (math.nan, -math.inf, False)])
@pytest.mark.parametrize("bound", [2e-3, math.inf])
def test_a_value_is_inside_its_bound_only_if_it_is_shown_to_be(got, want, fine, bound):
    fine = fine or (bound == math.inf and math.isfinite(got) and math.isfinite(want))
    g, w = torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.float64)
    g[1, 2], w[1, 2] = got, want
    if fine:
        ref.inside(g, w, torch.full_like(w, bound))
    else:
        with pytest.raises(AssertionError):
            ref.inside(g, w, torch.full_like(w, bound))


def test_the_definition_of_rows_that_see_infinities_and_nothing():
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(6, 2, 4, generator=g, dtype=torch.float64) for _ in range(3))
    mask = ref.sees(0, 6, 6, 3, 1)
    o, lse = ref.definition(q, k, v, mask)
    wo, wl, _, _ = ref.forward(q, k, v, mask, torch.float32)
    torch.testing.assert_close(o, wo, rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(lse, wl, rtol=1e-12, atol=1e-12)
    q[:, :, 0] = -q[:, :, 0].abs()
    k[0, :, 0] = math.inf                       # every row sees key 0: row 0 nothing else, the others with probability 0
    mask[4] = False
    o, lse = ref.definition(q, k, v, mask)
    assert bool(torch.isnan(o[0]).all()) and bool((lse[0] == -math.inf).all())
    assert not o[4].any() and bool((lse[4] == -math.inf).all())
    m2 = mask.clone()
    m2[:, 0] = False
    wo, wl = ref.definition(q[1:4], k, v, m2[1:4])
    torch.testing.assert_close(o[1:4], wo, rtol=1e-12, atol=1e-12)
    torch.testing.assert_close(lse[1:4], wl, rtol=1e-12, atol=1e-12)
