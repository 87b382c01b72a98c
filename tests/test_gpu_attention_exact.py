"""bf16 windowed and paged attention with head sizes 32 and 128: as exact as its outputs are rounded, as attention over whole sequences is
(test_gpu_kernels.py).  Probabilities and dS enter their products with at least 16 bits, rows are summed in fp32: all that is left of the error
is the rounding of the bf16 outputs, plus 2 % for operands (2^-17 against 2^-9) and single roundings that fall the other way."""
import pytest
import torch

import attention_reference as ref
import paper_2403_10616_amd as dp
from gpu_util import DEV
from test_gpu_paged import Cache, starts_of
from test_gpu_window import ALL, bwd, draw, fwd, heads_of

pytestmark = pytest.mark.gpu

HEADS = pytest.mark.parametrize("dh", [32, 128])


def as_exact_as_rounded(got, want, what):
    got, least = got.double().cpu(), (want.to(torch.bfloat16).double() - want).norm() / want.norm()
    err = (got - want).norm() / want.norm()
    print(f"  {what}: {float(err):.3e}, rounding {float(least):.3e}", flush=True)
    assert float(err) <= 1.02 * float(least), what


@HEADS
@pytest.mark.parametrize("B,S,H,Hkv,window,sinks,lengths", [
    (4, 33, 4, 4, ALL, 0, None), (2, 300, 4, 2, 65, 5, [300, 170]), (1, 1000, 2, 1, ALL, 0, None), (2, 700, 8, 1, 64, 3, None), (40, 200, 8, 4, 100, 2, None), (1, 1500, 4, 2, 900, 40, None)])
def test_windowed(dh, B, S, H, Hkv, window, sinks, lengths):
    """one and two groups of waves, blocks of 128 and of 32 keys, sinks whole and in parts"""
    print(f"exact window B={B} S={S} H={H} Hkv={Hkv} dh={dh} W={window} sinks={sinks} lengths={lengths}", flush=True)
    x, g = draw((B * S, (H + 2 * Hkv) * dh), 41, dp.BF16), draw((B * S, H * dh), 42, dp.BF16)
    rows = lengths or [S] * B
    len_d = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    o, lse = fwd(dp.BF16, x.to(DEV), len_d, B, S, H, Hkv, dh, window, sinks)
    d = bwd(dp.BF16, x.to(DEV), len_d, o, g.to(DEV), lse, B, S, H, Hkv, dh, window, sinks)
    parts = {name: ([], []) for name in ("o", "dq", "dk", "dv")}
    stored = o.double().cpu()
    for b in list(range(B))[:3]:
        n = rows[b]
        at = slice(b * S, b * S + n)
        q, k, v = heads_of(x[at], n, H, Hkv, dh)
        mask = ref.sees(0, n, n, window, sinks)
        wo, wl, _, _ = ref.forward(q, k, v, mask, torch.float32)
        grads = ref.backward(q, k, v, stored[at].reshape(n, H, dh), g[at].double().reshape(n, H, dh), wl, mask, torch.float32)[:3]
        have = heads_of(d[at], n, H, Hkv, dh)
        for name, a, w in zip(parts, (stored[at].reshape(n, H, dh), *have), (wo, *grads)):
            parts[name][0].append(a.cpu().reshape(-1))
            parts[name][1].append(w.reshape(-1))
        assert float((lse[b, :, :n].T.double().cpu() - wl).abs().max()) <= 1e-5
    for name, (a, w) in parts.items():
        as_exact_as_rounded(torch.cat(a), torch.cat(w), name)


@HEADS
@pytest.mark.parametrize("cached,new,H,Hkv,window,sinks", [
    ([100 + 17 * b for b in range(40)], [1] * 40, 16, 4, ALL, 0), ([3000, 1200, 2500, 40], [2, 1, 3, 1], 16, 2, ALL, 0), ([2000], [300], 4, 2, 900, 4), ([10, 0, 700], [130, 64, 200], 4, 4, ALL, 0),
    ([5000, 30], [3, 400], 8, 2, ALL, 0)])
def test_paged(dh, cached, new, H, Hkv, window, sinks):
    """few rows and blocks of many, of one and of several splits"""
    print(f"exact paged cached={cached} new={new} H={H} Hkv={Hkv} dh={dh} W={window} sinks={sinks}", flush=True)
    c = Cache(dp.BF16, [a + b for a, b in zip(cached, new)], Hkv, dh, 16, 3)
    st = starts_of(cached)
    c.append(draw((st[-1], (H + 2 * Hkv) * dh), 43, dp.BF16).to(DEV), st, [0] * len(cached), H)
    st = starts_of(new)
    x = draw((st[-1], (H + 2 * Hkv) * dh), 44, dp.BF16)
    c.append(x.to(DEV), st, cached, H)
    o, lse = c.attend(x.to(DEV), st, cached, H, max(new), window, sinks)
    want = torch.zeros((st[-1], H, dh), dtype=torch.float64)
    for b, (m, n) in enumerate(zip(cached, new)):
        kv = c.kv[b].double()
        wo, wl, _, _ = ref.forward(heads_of(x[st[b]:st[b + 1]], n, H, Hkv, dh)[0], kv[:, 0], kv[:, 1], ref.sees(m, n, m + n, window, sinks), torch.float32)
        want[st[b]:st[b + 1]] = wo
        assert float((lse[st[b]:st[b + 1]].double().cpu() - wl).abs().max()) <= 1e-5
    as_exact_as_rounded(o.reshape(-1, H, dh), want, "o")
