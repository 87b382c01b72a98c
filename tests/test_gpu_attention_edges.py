"""Windowed and paged attention once more with `attention_reference.inside`, which no NaN passes, and batches of more documents than one wave
looks through at once or one launch takes."""
import random

import pytest
import torch

import attention_reference as ref
import paper_2403_10616_amd as dp
import test_gpu_paged
import test_gpu_window
from gpu_util import DEV
from test_gpu_window import ALL, TDT, draw, fwd, heads_of, scratch

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [dp.F32, dp.BF16])


@pytest.fixture
def strict(monkeypatch):
    monkeypatch.setattr(test_gpu_window, "within", ref.inside)
    monkeypatch.setattr(test_gpu_paged, "within", ref.inside)


# ---- no NaN passes ------------------------------------------------------------------------------------------------------
@TYPES
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_windows_with_no_nan_let_through(strict, dtype, dh):
    test_gpu_window.check(dtype, 2, 300, 4, 2, dh, 65, 70, [300, 130])


@TYPES
@pytest.mark.parametrize("dh", [32, 64, 128])
def test_chunks_and_tokens_with_no_nan_let_through(strict, dtype, dh):
    test_gpu_paged.check(dtype, [300, 0, 2000, 5], [40, 33, 1, 128], 4, 1, dh, 16, ALL, 0)


@TYPES
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 2, 70]])
def test_pages_that_are_gone_let_no_nan_through(strict, dtype, new):
    test_gpu_paged.test_pages_that_are_gone_hold_no_keys(dtype, new)


def test_pages_beyond_32_bits_let_no_nan_through(strict):
    test_gpu_paged.test_offsets_beyond_32_bits()


# ---- many documents -----------------------------------------------------------------------------------------------------
@TYPES
@pytest.mark.parametrize("H,Hkv,dh", [(2, 1, 32), (3, 3, 64), (8, 2, 128)])
def test_chunks_among_many_documents(strict, dtype, H, Hkv, dh):
    """150 documents, which a wave looks through 64 at a time: chunks among the first, the middle and the last ones, beside tokens and nothing"""
    rng = random.Random(11 * H)
    new = [rng.choice([0, 1, rng.randint(40, 200)]) if b % 3 else rng.randint(0, 2) for b in range(150)]
    new[0] = new[63] = new[64] = new[127] = new[128] = new[149] = 65
    assert all(sum(n > 32 for n in new[a:b]) >= 4 for a, b in ((0, 64), (64, 128), (128, 150)))
    test_gpu_paged.check(dtype, [rng.randint(0, 90) for _ in new], new, H, Hkv, dh, 16, rng.choice([ALL, 70]), 3, seed=12)


def filled(shape, dtype, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=TDT[dtype], device=DEV).normal_(generator=g)


@TYPES
def test_a_batch_of_more_documents_than_one_launch_takes(dtype):
    """131072 documents of 8 heads and up to 64 rows are one launch of the windowed calls; 300 more are another.  All documents against two calls of
    half of them each, bit for bit, and those around the cut against 64 bits"""
    B, S, H, Hkv, dh, window, sinks = (1 << 17) + 300, 3, 8, 1, 32, 2, 1
    print(f"documents in parts dtype={dtype}", flush=True)
    x, g = filled((B * S, (H + 2 * Hkv) * dh), dtype, 1), filled((B * S, H * dh), dtype, 2)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    lengths = torch.randint(0, S + 1, (B,), device=DEV, generator=gen, dtype=torch.int32)
    dsum = scratch(B, H, S)

    def both(lo, hi):
        at, n = slice(lo * S, hi * S), hi - lo
        o, lse = fwd(dtype, x[at], lengths[lo:hi], n, S, H, Hkv, dh, window, sinks)
        d = torch.full_like(x[at], 77.0)
        dp.dipaco_k_attention_window_bwd(dtype, x[at], lengths[lo:hi], o, g[at], lse, d, dsum, n, S, H, Hkv, dh, window, sinks)
        return o, lse, d

    o, lse, d = both(0, B)
    half = B // 8 * 4                        # integers begin at 16 bytes
    for lo, hi in ((0, half), (half, B)):
        for whole, part in zip((o, lse, d), both(lo, hi)):
            rows = S if whole.shape[0] == B * S else 1
            assert torch.equal(whole[lo * rows:hi * rows], part)
    for b in (0, 1, half, (1 << 17) - 2, (1 << 17) - 1, 1 << 17, (1 << 17) + 1, B - 1):
        n = int(lengths[b])
        at = slice(b * S, b * S + n)
        assert not o[b * S + n:(b + 1) * S].any() and not lse[b, :, n:].any() and not d[b * S + n:(b + 1) * S].any()
        if not n:
            continue
        q, k, v = heads_of(x[at].cpu(), n, H, Hkv, dh)
        mask = ref.sees(0, n, n, window, sinks)
        wo, wl, eo, el = ref.forward(q, k, v, mask, TDT[dtype])
        ref.inside(o[at].reshape(n, H, dh), wo, eo, f"o[{b}]")
        ref.inside(lse[b, :, :n].T, wl, el, f"lse[{b}]")
        res = ref.backward(q, k, v, o[at].double().cpu().reshape(n, H, dh), g[at].double().cpu().reshape(n, H, dh), lse[b, :, :n].T.double().cpu(), mask, TDT[dtype])
        for name, got, w, e in zip(("dq", "dk", "dv"), heads_of(d[at].cpu(), n, H, Hkv, dh), res[:3], res[3:]):
            ref.inside(got, w, e, f"{name}[{b}]")


def attend_all(dtype, x, row_start, cache_len, pages, cache, max_new, H, Hkv, dh, page, window, sinks):
    T, B, per_doc = x.shape[0], cache_len.numel(), pages.shape[1]
    dp.dipaco_k_cache_append(dtype, x, row_start, cache_len, pages, cache, T, B, H, Hkv, dh, cache.shape[0], page, per_doc)
    o, lse = torch.full((T, H * dh), 77.0, dtype=TDT[dtype], device=DEV), torch.full((T, H), 77.0, device=DEV)
    ws = torch.empty(dp.dipaco_k_attention_paged_workspace_bytes(T, B, max_new, H, Hkv, dh, page, per_doc), dtype=torch.uint8, device=DEV)
    dp.dipaco_k_attention_paged(dtype, x, row_start, cache_len, pages, cache, o, lse, T, B, max_new, H, Hkv, dh, cache.shape[0], page, per_doc, window, sinks, ws)
    return o, lse


def check_documents(dtype, docs, x, row_start, cache_len, pages, cache, o, lse, H, Hkv, dh, page, window, sinks):
    for b in docs:
        lo, hi, m = int(row_start[b]), int(row_start[b + 1]), int(cache_len[b])
        n = hi - lo
        if not n:
            continue
        kv = torch.cat([cache[p] for p in pages[b].tolist()], 2).double().cpu().permute(2, 0, 1, 3)[:m + n]
        wo, wl, eo, el = ref.forward(heads_of(x[lo:hi].cpu(), n, H, Hkv, dh)[0], kv[:, 0], kv[:, 1], ref.sees(m, n, m + n, window, sinks), TDT[dtype])
        ref.inside(o[lo:hi].reshape(n, H, dh), wo, eo, f"o[{b}]")
        ref.inside(lse[lo:hi], wl, el, f"lse[{b}]")


@TYPES
def test_tokens_of_more_documents_than_a_grid_is_deep(dtype):
    """a token each for 65535 + 70 documents on pages of 16: a second launch from document 65535 on"""
    B, H, Hkv, dh, page = 65535 + 70, 2, 1, 32, 16
    print(f"tokens of {B} documents dtype={dtype}", flush=True)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(4)
    x, cache = filled((B, (H + 2 * Hkv) * dh), dtype, 5), filled((B, 2, Hkv, page, dh), dtype, 6)
    pages = torch.randperm(B, device=DEV, generator=gen).int().reshape(B, 1)
    cache_len = torch.randint(0, page, (B,), device=DEV, generator=gen, dtype=torch.int32)
    row_start = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    o, lse = attend_all(dtype, x, row_start, cache_len, pages, cache, 1, H, Hkv, dh, page, 9, 1)
    check_documents(dtype, [0, 1, 40000, *range(65525, 65545), *range(B - 10, B)], x, row_start, cache_len, pages, cache, o, lse, H, Hkv, dh, page, 9, 1)
    half = B // 8 * 4                                                                        # and all of them against two calls; integers begin at 16 bytes
    for at in (slice(0, half), slice(half, B)):
        n = at.stop - at.start
        got = attend_all(dtype, x[at].contiguous(), row_start[:n + 1], cache_len[at].contiguous(), pages[at].contiguous(), cache, 1, H, Hkv, dh, page, 9, 1)
        assert torch.equal(got[0], o[at]) and torch.equal(got[1], lse[at])


def test_more_chunks_than_a_grid_is_deep():
    """fp32, 13300 documents of 40 tokens of 8 heads on one: five blocks of 64 packed rows each, a second launch from block 65535 (document 13107) on"""
    dtype, B, n, H, Hkv, dh, page, per_doc = dp.F32, 13300, 40, 8, 1, 32, 16, 4
    print(f"chunks of {B} documents", flush=True)
    assert B * (n * H // 64) > 65535
    gen = torch.Generator(device=DEV)
    gen.manual_seed(7)
    x, cache = filled((B * n, (H + 2 * Hkv) * dh), dtype, 8), filled((B * per_doc, 2, Hkv, page, dh), dtype, 9)
    pages = torch.randperm(B * per_doc, device=DEV, generator=gen).int().reshape(B, per_doc)
    cache_len = torch.randint(0, per_doc * page - n, (B,), device=DEV, generator=gen, dtype=torch.int32)
    row_start = n * torch.arange(B + 1, dtype=torch.int32, device=DEV)
    o, lse = attend_all(dtype, x, row_start, cache_len, pages, cache, n, H, Hkv, dh, page, ALL, 0)
    check_documents(dtype, [0, 1, 7000, *range(13100, 13115), B - 1], x, row_start, cache_len, pages, cache, o, lse, H, Hkv, dh, page, ALL, 0)
    half = B // 8 * 4                        # integers begin at 16 bytes
    for at in (slice(0, half), slice(half, B)):
        m = at.stop - at.start
        rows = slice(at.start * n, at.stop * n)
        got = attend_all(dtype, x[rows], row_start[:m + 1], cache_len[at].contiguous(), pages[at].contiguous(), cache, n, H, Hkv, dh, page, ALL, 0)
        assert torch.equal(got[0], o[rows]) and torch.equal(got[1], lse[rows])
