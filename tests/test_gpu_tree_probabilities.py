"""Attention of trees in bf16 against 64 bits: no more is lost than the output's own rounding and 2^-17 of each probability, for every head size.

A score is off by at most dh u times the sum of its products' magnitudes (u = 2^-24), its exponential by that much relative to itself and 32 u; n terms
add n u (attention_reference.py).  A probability held in 16 bits is off by 2^-17 of itself at most, and the output is rounded once, by half a step."""
import math
import random

import pytest
import torch

import attention_reference as aref
import draft_reference as ref
import paper_2403_10616_amd as dp
from test_gpu_drafts import tree
from test_gpu_tree_attention import attend, filled, mask_of
from test_gpu_window import ALL, TDT, heads_of
from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("cached,counts,H,Hkv,window", [
    ([0, 3], [9, 16], 2, 2, ALL), ([1000], [16], 14, 14, ALL), ([900, 40], [64, 100], 4, 2, 300), ([5000, 30], [40, 64], 4, 1, ALL), ([3000], [400], 2, 1, 2048)])
def test_probabilities_keep_16_bits(dh, cached, counts, H, Hkv, window):
    page, sinks = 16, 2
    c, x, st = filled(dp.BF16, cached, counts, H, Hkv, dh, page, 17)
    parents = [ref.random_parents(random.Random(b), k, "level") for b, k in enumerate(counts)]
    depth, seen = tree(parents)
    o, _ = attend(c, x.to(DEV), st, cached, depth, seen, H, max(counts), window, sinks)
    scale, h = 1.0 / math.sqrt(dh), aref.half_step(TDT[dp.BF16])
    for b, (m, k) in enumerate(zip(cached, counts)):
        rows = ref.seen_rows(parents[b])
        mask = mask_of(m, rows, [len(r) - 1 for r in rows], window, sinks, m + k)
        kv, q = c.kv[b].double(), heads_of(x[st[b]:st[b + 1]], k, H, Hkv, dh)[0]
        for y in range(H):
            kk, vv = kv[:, 0, y * Hkv // H], kv[:, 1, y * Hkv // H]
            p = torch.softmax((q[:, y] @ kk.T * scale).masked_fill(~mask, -math.inf), 1)
            size = (q[:, y].abs() @ kk.abs().T * scale).masked_fill(~mask, 0.0).amax(1)
            rel = aref.U * (2 * dh * size + mask.sum(1) + 32) + 2.0 ** -17
            want = p @ vv
            aref.inside(o[st[b]:st[b + 1]].reshape(k, H, dh)[:, y], want, 2 * rel[:, None] * (p @ vv.abs()) + h * want.abs(), f"o[{b}], head {y}")
