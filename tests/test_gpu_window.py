"""Attention with a sliding window and sinks against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2403_10616_amd as dp
from gpu_util import DEV

pytestmark = pytest.mark.gpu

TDT = {dp.F32: torch.float32, dp.BF16: torch.bfloat16}
ALL = 1 << 30


def draw(shape, seed, dtype, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(TDT[dtype])


def scratch(B, H, S):
    return torch.full((2 * B * H * ((S + 127) // 128 * 128),), float("nan"), device=DEV)


def fwd(dtype, qkv, lengths, B, S, H, Hkv, dh, window, sinks, stream=None):
    o = torch.full((B * S, H * dh), 77.0, dtype=TDT[dtype], device=DEV)
    lse = torch.full((B, H, S), 77.0, device=DEV)
    dp.dipaco_k_attention_window_fwd(dtype, qkv, lengths, o, lse, B, S, H, Hkv, dh, window, sinks, stream=stream)
    return o, lse


def bwd(dtype, qkv, lengths, o, d_o, lse, B, S, H, Hkv, dh, window, sinks):
    dqkv = torch.full_like(qkv, 77.0)
    dp.dipaco_k_attention_window_bwd(dtype, qkv, lengths, o, d_o, lse, dqkv, scratch(B, H, S), B, S, H, Hkv, dh, window, sinks)
    return dqkv


def heads_of(x, n, H, Hkv, dh):
    return [p.double().reshape(n, p.shape[1] // dh, dh) for p in (x[:, :H * dh], x[:, H * dh:(H + Hkv) * dh], x[:, (H + Hkv) * dh:])]


def within(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    over = err > bound + 1e-30
    assert not bool(over.any()), f"{what}: {int(over.sum())} of {over.numel()} out of bounds, worst {float((err / (bound + 1e-30)).max()):.2f} x"
    print(f"  {what}: worst {float((err / (bound + 1e-30)).max()):.2f} of its bound", flush=True)


def check(dtype, B, S, H, Hkv, dh, window, sinks, lengths=None, seed=1, scale=1.0):
    print(f"window dtype={dtype} B={B} S={S} H={H} Hkv={Hkv} dh={dh} W={window} sinks={sinks} lengths={lengths}", flush=True)
    t = TDT[dtype]
    x = draw((B * S, (H + 2 * Hkv) * dh), seed, dtype, scale)
    g = draw((B * S, H * dh), seed + 1, dtype)
    rows = [S] * B if lengths is None else [min(max(n, 0), S) for n in lengths]
    for b, n in enumerate(rows):                               # what lies behind a document is not read
        x[b * S + n:(b + 1) * S] = float("nan")
        g[b * S + n:(b + 1) * S] = float("nan")
    len_d = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    xd, gd = x.to(DEV), g.to(DEV)
    o, lse = fwd(dtype, xd, len_d, B, S, H, Hkv, dh, window, sinks)
    o_in, lse_in = torch.full((B * S, H * dh), float("nan"), dtype=t), torch.full((B, H, S), float("nan"))
    want = []
    for b, n in enumerate(rows):
        at = slice(b * S, b * S + n)
        assert not o[b * S + n:(b + 1) * S].any() and not lse[b, :, n:].any()      # zeros behind it
        if not n:
            want.append(None)
            continue
        q, k, v = heads_of(x[at], n, H, Hkv, dh)
        mask = ref.sees(0, n, n, window, sinks)
        wo, wl, eo, el = ref.forward(q, k, v, mask, t)
        within(o[at].reshape(n, H, dh), wo, eo, f"o[{b}]")
        within(lse[b, :, :n].T, wl, el, f"lse[{b}]")
        o_in[at], lse_in[b, :, :n] = wo.reshape(n, -1).to(t), wl.T.float()
        want.append((q, k, v, mask))
    dqkv = bwd(dtype, xd, len_d, o_in.to(DEV), gd, lse_in.to(DEV), B, S, H, Hkv, dh, window, sinks)
    for b, n in enumerate(rows):
        assert not dqkv[b * S + n:(b + 1) * S].any()
        if not n:
            continue
        at = slice(b * S, b * S + n)
        q, k, v, mask = want[b]
        res = ref.backward(q, k, v, o_in[at].double().reshape(n, H, dh), g[at].double().reshape(n, H, dh), lse_in[b, :, :n].T.double(), mask, t)
        for name, got, w, e in zip(("dq", "dk", "dv"), heads_of(dqkv[at], n, H, Hkv, dh), res[:3], res[3:]):
            within(got, w, e, f"{name}[{b}]")
    o2, lse2 = fwd(dtype, xd, len_d, B, S, H, Hkv, dh, window, sinks)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)                            # the same bits again
    assert torch.equal(dqkv, bwd(dtype, xd, len_d, o_in.to(DEV), gd, lse_in.to(DEV), B, S, H, Hkv, dh, window, sinks))


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("S,window,sinks", [(1, 1, 0), (2, 1, 1), (33, 7, 0), (64, 64, 0), (65, 64, 1), (130, 1, 0), (130, 1, 3), (257, 33, 5), (300, 65, 70),
                                            (300, 130, 0), (190, ALL, 0), (190, ALL, 7), (190, 20, ALL)])
def test_sizes_windows_and_sinks(dtype, dh, S, window, sinks):
    check(dtype, 1, S, 2, 1, dh, window, sinks)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks", [(3, 70, 6, 2, 32, 20, 2), (2, 129, 8, 8, 64, 40, 0), (2, 200, 5, 1, 64, 64, 4), (1, 260, 8, 1, 128, 100, 16),
                                                       (2, 515, 3, 3, 64, 129, 1), (1, 1030, 2, 1, 64, 256, 4)])
def test_heads_that_share_keys(dtype, B, S, H, Hkv, dh, window, sinks):
    check(dtype, B, S, H, Hkv, dh, window, sinks, seed=5)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("dh,S,lengths,window,sinks", [(64, 100, [100, 0, 1, 37], 16, 2), (32, 140, [0, 0, 140], ALL, 0), (128, 200, [129, 128, 127, 64, 65], 30, 3),
                                                       (64, 64, [-5, 900, 63], 8, 1), (64, 1, [0, 1], 1, 0)])
def test_padded_batches(dtype, dh, S, lengths, window, sinks):
    check(dtype, len(lengths), S, 4, 2, dh, window, sinks, lengths, seed=7)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,lengths", [(1, 1700, 1, 1, 64, 100, 5, None), (2, 1000, 8, 2, 32, 64, 40, [1000, 130]), (1, 1300, 4, 1, 128, 200, 3, None),
                                                               (3, 900, 6, 2, 64, 33, 33, [900, 20, 500]), (1, 800, 16, 1, 32, 10, 1, None), (1, 600, 8, 1, 64, 1, 600, None)])
def test_sinks_of_documents_that_are_much_longer_than_the_window(dtype, B, S, H, Hkv, dh, window, sinks, lengths):
    """the sinks' gradients are sums over all rows behind them, cut into parts where there are many"""
    check(dtype, B, S, H, Hkv, dh, window, sinks, lengths, seed=13)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
def test_peaked_rows(dtype):
    """scores of +-60: the running maximum moves by more than an fp32 exponential's range holds in probabilities"""
    check(dtype, 1, 400, 2, 2, 64, 150, 4, seed=9, scale=4.0)


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("dh,S,H", [(64, 300, 2), (32, 100, 2), (128, 140, 1)])
def test_a_window_over_everything_is_causal_attention(dtype, dh, S, H):
    """the same formula as dipaco_k_attention_fwd / _bwd: both are within a rounding of the output of each other, and of fp32's sums"""
    x = draw((S, 3 * H * dh), 11, dtype).to(DEV)
    g = draw((S, H * dh), 12, dtype).to(DEV)
    o, lse = fwd(dtype, x, None, 1, S, H, H, dh, S, 0)
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    dp.dipaco_k_attention_fwd(dtype, x, o2, lse2, 1, S, H, dh)
    d = bwd(dtype, x, None, o, g, lse, 1, S, H, H, dh, S, 0)
    d2 = torch.empty_like(d)
    dp.dipaco_k_attention_bwd(dtype, x, o, g, lse, d2, scratch(1, H, S), 1, S, H, dh)
    tol = 2e-5 if dtype == dp.F32 else 1e-2
    for a, b in ((o, o2), (lse, lse2), (d, d2)):
        assert float((a.double() - b.double()).norm() / b.double().norm()) <= tol


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("where,value", [("q", float("nan")), ("k", float("inf")), ("k", float("nan")), ("v", float("nan")), ("v", float("-inf")), ("g", float("inf"))])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(dtype, dh, where, value):
    S, H, Hkv, window, sinks, at = 150, 2, 1, 40, 3, 70
    print(f"not finite dtype={dtype} dh={dh} {where}={value}", flush=True)
    x, g = draw((S, (H + 2 * Hkv) * dh), 21, dtype), draw((S, H * dh), 22, dtype)
    col = {"q": 1, "k": H * dh + 1, "v": (H + Hkv) * dh + 1, "g": 1}[where]       # of head 0, or of the keys' only head
    clean_o, clean_lse = fwd(dtype, x.to(DEV), None, 1, S, H, Hkv, dh, window, sinks)
    clean = bwd(dtype, x.to(DEV), None, clean_o, g.to(DEV), clean_lse, 1, S, H, Hkv, dh, window, sinks)
    (g if where == "g" else x)[at, col] = value
    o, lse = fwd(dtype, x.to(DEV), None, 1, S, H, Hkv, dh, window, sinks)
    d = bwd(dtype, x.to(DEV), None, o, g.to(DEV), lse, 1, S, H, Hkv, dh, window, sinks)
    seen = ref.sees(0, S, S, window, sinks)
    rows = torch.zeros((S, H), dtype=torch.bool)                                   # (row, head) whose o the value reaches
    if where == "q":
        rows[at, 0] = True
    elif where in "kv":
        rows |= seen[:, at][:, None]
    o_h, clean_h = o.reshape(S, H, dh).cpu(), clean_o.reshape(S, H, dh).cpu()
    # what is reached is not finite (a column of a value, all columns of a score); what is not keeps a result within rounding of its own
    for r in range(S):
        for h in range(H):
            if not rows[r, h]:
                assert bool(torch.isfinite(o_h[r, h]).all()), (r, h)
                assert float((o_h[r, h].double() - clean_h[r, h].double()).abs().max()) <= 4 * ref.half_step(TDT[dtype]) * float(clean_h[r, h].abs().max()) + 1e-5
            elif where == "v":
                assert not bool(torch.isfinite(o_h[r, h, 1]))
            elif value != value:
                assert bool(torch.isnan(o_h[r, h]).all())
    # gradients: rows whose o was reached, and for g its own row, pass it on to the keys that they see
    bad = rows.clone()
    if where == "g":
        bad[at, 0] = True
    keys = (seen.double().T @ bad.any(1).double()) > 0
    dq, dk, dv = (p.reshape(S, -1, dh) for p in (d[:, :H * dh].cpu(), d[:, H * dh:(H + Hkv) * dh].cpu(), d[:, (H + Hkv) * dh:].cpu()))
    cq, ck, cv = (p.reshape(S, -1, dh) for p in (clean[:, :H * dh].cpu(), clean[:, H * dh:(H + Hkv) * dh].cpu(), clean[:, (H + Hkv) * dh:].cpu()))
    tol = 16 * ref.half_step(TDT[dtype])
    for r in range(S):
        for h in range(H):
            if not bad[r, h]:
                assert bool(torch.isfinite(dq[r, h]).all()), ("dq", r, h)
                assert float((dq[r, h].double() - cq[r, h].double()).abs().max()) <= tol * float(cq[r, h].abs().max()) + 1e-4
        if not keys[r]:
            for name, a, c in (("dk", dk, ck), ("dv", dv, cv)):
                assert bool(torch.isfinite(a[r]).all()), (name, r)
                assert float((a[r].double() - c[r].double()).abs().max()) <= tol * float(c[r].abs().max()) + 1e-4


def test_gradient_against_differences():
    """d/dt of sum(w * o(x + t y)) by differences of the fp32 forward pass: a step of 1e-2 leaves an error of the order of 1e-4 of the
    slope (the third derivative) and 2^-24 * sqrt(values) / 1e-2 of rounding"""
    B, S, H, Hkv, dh, window, sinks, lengths = 2, 90, 4, 2, 32, 25, 2, [90, 41]
    x, y = draw((B * S, (H + 2 * Hkv) * dh), 31, dp.F32).to(DEV), draw((B * S, (H + 2 * Hkv) * dh), 32, dp.F32).to(DEV)
    w = draw((B * S, H * dh), 33, dp.F32).to(DEV)
    len_d = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    o, lse = fwd(dp.F32, x, len_d, B, S, H, Hkv, dh, window, sinks)
    d = bwd(dp.F32, x, len_d, o, w, lse, B, S, H, Hkv, dh, window, sinks)
    slope = float((d.double() * y.double()).sum())
    e = 1e-2
    up, down = (fwd(dp.F32, x + s * e * y, len_d, B, S, H, Hkv, dh, window, sinks)[0].double() for s in (1, -1))
    got = float(((up - down) * w.double()).sum() / (2 * e))
    assert abs(got - slope) <= 2e-3 * float((d.double() * y.double()).norm()), (got, slope)


def test_captured_and_replayed_beside_eager_work():
    dtype, B, S, H, Hkv, dh, window, sinks = dp.BF16, 2, 200, 4, 2, 64, 50, 4
    x, g = draw((B * S, (H + 2 * Hkv) * dh), 41, dtype).to(DEV), draw((B * S, H * dh), 42, dtype).to(DEV)
    lengths = torch.tensor([200, 90], dtype=torch.int32, device=DEV)
    o, lse, d, ds = (torch.empty((B * S, H * dh), dtype=TDT[dtype], device=DEV), torch.empty((B, H, S), device=DEV), torch.empty_like(x), scratch(B, H, S))
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        dp.dipaco_k_attention_window_fwd(dtype, x, lengths, o, lse, B, S, H, Hkv, dh, window, sinks)
        dp.dipaco_k_attention_window_bwd(dtype, x, lengths, o, g, lse, d, ds, B, S, H, Hkv, dh, window, sinks)
    for k in range(4):
        x.copy_(draw(tuple(x.shape), 50 + k, dtype))
        lengths.copy_(torch.tensor([200 - 30 * k, 40 * k], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        eo, el = fwd(dtype, x, lengths, B, S, H, Hkv, dh, window, sinks)
        assert torch.equal(eo, o) and torch.equal(el, lse)
        assert torch.equal(bwd(dtype, x, lengths, eo, g, el, B, S, H, Hkv, dh, window, sinks), d)


def test_on_a_stream_of_its_own():
    dtype, B, S, H, Hkv, dh = dp.BF16, 1, 500, 2, 2, 64
    x = draw((B * S, (H + 2 * Hkv) * dh), 61, dtype).to(DEV)
    want = fwd(dtype, x, None, B, S, H, Hkv, dh, 100, 0)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()) as _:
        got = fwd(dtype, x, None, B, S, H, Hkv, dh, 100, 0)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])
@pytest.mark.parametrize("dh", [32, 128])
def test_a_value_that_is_not_finite_behind_the_sinks(dtype, dh):
    """sinks whose gradients are cut into parts: a NaN in a row's gradient reaches the sinks, which the row sees, and its window, nothing else"""
    S, H, Hkv, window, sinks, at = 900, 8, 1, 40, 3, 500
    print(f"not finite behind the sinks dtype={dtype} dh={dh}", flush=True)
    x, g = draw((S, (H + 2 * Hkv) * dh), 23, dtype).to(DEV), draw((S, H * dh), 24, dtype).to(DEV)
    o, lse = fwd(dtype, x, None, 1, S, H, Hkv, dh, window, sinks)
    clean = bwd(dtype, x, None, o, g, lse, 1, S, H, Hkv, dh, window, sinks)[:, H * dh:]
    g[at, 0] = float("nan")
    d = bwd(dtype, x, None, o, g, lse, 1, S, H, Hkv, dh, window, sinks)
    reached = ref.sees(0, S, S, window, sinks)[at].to(DEV)
    keys = d[:, H * dh:]
    assert bool(torch.isnan(keys[reached][:, :Hkv * dh]).all()) and bool(torch.isnan(keys[reached][:, Hkv * dh]).all())
    assert bool(torch.isnan(d[at, :dh]).all()) and int(torch.isnan(d[:, :H * dh]).sum()) == dh
    tol = 16 * ref.half_step(TDT[dtype])
    rest = (keys[~reached].double() - clean[~reached].double()).abs()
    assert bool((rest <= tol * clean[~reached].double().abs().amax(1, keepdim=True) + 1e-4).all())


@pytest.mark.parametrize("B,S,H,Hkv,dh,window,sinks,lengths", [(1, 700, 2, 2, 64, ALL, 0, None), (2, 450, 3, 1, 32, ALL, 0, [450, 100]), (1, 900, 2, 1, 128, 400, 9, None),
                                                               (40, 449, 2, 2, 64, ALL, 0, None), (20, 400, 14, 7, 64, 300, 2, None)])
def test_blocks_of_one_and_of_two_groups_of_waves(B, S, H, Hkv, dh, window, sinks, lengths):
    """few long blocks (two groups of waves a block, 32 keys a workgroup in the gradient) and enough of them"""
    check(dp.BF16, B, S, H, Hkv, dh, window, sinks, lengths, seed=15)


def test_offsets_beyond_32_bits():
    """a batch whose rows lie beyond 2^32 bytes and 2^31 elements of qkv: the last document, bit for bit as it is alone"""
    dtype, B, S, H, Hkv, dh, window = dp.BF16, 6, 65536, 16, 16, 128, 100
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = torch.empty((B * S, (H + 2 * Hkv) * dh), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    d_o = torch.empty((B * S, H * dh), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    assert x.numel() > 1 << 31
    o, lse = fwd(dtype, x, None, B, S, H, Hkv, dh, window, 0)
    d = bwd(dtype, x, None, o, d_o, lse, B, S, H, Hkv, dh, window, 0)
    for b in (0, B - 1):
        at = slice(b * S, (b + 1) * S)
        o1, lse1 = fwd(dtype, x[at].contiguous(), None, 1, S, H, Hkv, dh, window, 0)
        assert torch.equal(o[at], o1) and torch.equal(lse[b], lse1[0])
        d1 = bwd(dtype, x[at].contiguous(), None, o1, d_o[at].contiguous(), lse1, 1, S, H, Hkv, dh, window, 0)
        assert torch.equal(d[at], d1)
        assert bool(torch.isfinite(d1).all()) and float(d1.float().abs().amax()) > 0
