"""Drafted decoding step after step, each piece of every step held to its definition: positions and bits, attention in 64 bits over what the caches should hold, the walk on
the logits that the step made, and the caches that it leaves.  Nothing here hangs on a score that two roundings may decide differently."""
import random

import pytest
import torch

import attention_reference as aref
import draft_reference as ref
from test_gpu_drafts import TYPES
from test_gpu_paged import Cache, i32, starts_of
from test_gpu_tree_attention import Step, mask_of
from test_gpu_window import TDT, heads_of
import paper_2403_10616_amd as dp

pytestmark = pytest.mark.gpu

WINDOW, SINKS = 200, 4                                              # Step's


class Sampled(Step):
    """a step that draws at a temperature"""
    temperature = 0.0

    def run(self):
        T, B, n, c = self.T, self.B, self.n, self.c[0]
        dp.dipaco_k_draft_tree(self.parent, self.row_start, self.depth, self.seen, T, B, n)
        width = self.H * self.dh
        for l in range(self.layers):
            self.qkv[l].copy_(self.layer_inputs(l, self.tokens))
            dp.dipaco_k_cache_append(self.dtype, self.qkv[l], self.row_start, self.cache_len, self.pages, self.c[l].data, T, B, self.H, self.Hkv, self.dh, c.n_pages,
                                     self.page, c.per_doc)
            dp.dipaco_k_attention_tree(self.dtype, self.qkv[l], self.row_start, self.cache_len, self.depth, self.seen, self.pages, self.c[l].data, self.o[l], None, T, B,
                                       n, self.H, self.Hkv, self.dh, c.n_pages, self.page, c.per_doc, WINDOW, SINKS, self.ws)
            self.out[:, l * width:(l + 1) * width].copy_(self.o[l])
        self.logits(T, self.out, self.target)
        dp.dipaco_k_draft_verify(dp.F32, self.target, None, self.tokens, self.parent, self.row_start, self.u, self.v, self.path, self.kept, self.next, T, B, n, self.V,
                                 self.temperature, 1.0, False, self.vws)
        dp.dipaco_k_cache_keep(self.dtype, self.path, self.kept, self.cache_len, self.pages, [x.data for x in self.c], B, n, self.Hkv, self.dh, c.n_pages, self.page,
                               c.per_doc)
        self.cache_len += self.kept


def continuation(s, caches, done, fed, count):
    """`count` tokens behind each text, one by one; `fed`: how many tokens of each text the caches hold as they are"""
    for at in range(min(fed), max(len(t) for t in done) - 1):       # a document that is through writes its last one again
        s.one(caches, [t[:min(max(at, f) + 1, len(t))] for t, f in zip(done, fed)])
    texts = [list(t) for t in done]
    for _ in range(count):
        for b, x in enumerate(s.one(caches, texts)):
            texts[b].append(int(x.argmax()))
    return [t[len(d):] for t, d in zip(texts, done)]


@TYPES
@pytest.mark.parametrize("temperature", [0.0, 0.8])
def test_every_step_is_what_its_pieces_define(dtype, temperature):
    B, n, steps = 4, 12, 5
    s = Sampled(dtype, B, n)
    s.temperature = temperature
    plain = [Cache(dtype, [300] * B, s.Hkv, s.dh, s.page, 9) for _ in range(s.layers)]
    for c in plain:
        c.data.zero_()
    rng, g = random.Random(2), torch.Generator().manual_seed(3)
    tables = [t.cpu() for t in s.table]
    # texts of some length, so that the window leaves positions behind
    done = [[rng.randrange(s.V) for _ in range(k)] for k in (1, 205, 40, 190)]
    for l, c in enumerate(s.c):
        held = [t[:-1] for t in done]
        flat = torch.tensor([x for t in held for x in t], device=s.table[l].device)
        c.append(s.table[l][flat], starts_of([len(t) for t in held]), [0] * B, s.H)
    s.cache_len.copy_(i32([len(t) - 1 for t in done]))
    fed, longest = [0] * B, 0
    for step in range(steps):
        right = continuation(s, plain, done, fed, n)
        fed = [len(t) - 1 for t in done]
        parents, tokens, counts = [], [], []
        for b in range(B):
            k = n if (step + b) % 4 else (step + b) % 8 // 4        # now and then a document has one row, or none
            p, at, t = ref.random_parents(rng, k, rng.choice(["level", "deep", "chain"])), {0: 0}, []
            for i in range(k):
                up = ref.parent_of(p[i], i)
                good = up in at and up >= 0
                t.append(done[b][-1] if i == 0 else right[b][at[up]] if good and rng.random() < 0.8 else rng.randrange(s.V))
                if i and good and t[i] == right[b][at[up]]:
                    at[i] = at[up] + 1
            parents.append(p)
            tokens.append(t)
            counts.append(k)
        st = starts_of(counts)
        pad = [0] * (s.T - st[-1])
        s.tokens.copy_(i32([x for t in tokens for x in t] + pad))
        s.parent.copy_(i32([x for p in parents for x in p] + pad))
        s.row_start.copy_(i32(st))
        u, v = torch.rand(s.T, generator=g) * 0.01, torch.rand(B, generator=g)
        s.u.copy_(u)
        s.v.copy_(v)
        s.run()
        depth, seen, target, outs = s.depth.tolist(), s.seen.tolist(), s.target.cpu(), [o.cpu() for o in s.o]
        path, kept, token, cached = s.path.tolist(), s.kept.tolist(), s.next.tolist(), s.cache_len.tolist()
        for b in range(B):
            k, m, at = counts[b], len(done[b]) - 1, slice(st[b], st[b + 1])
            if k == 0:
                assert kept[b] == 0 and token[b] == -1 and path[b] == [-1] * n and cached[b] == m
                continue
            rows = ref.seen_rows(parents[b])
            assert depth[at] == [len(r) - 1 for r in rows] and seen[at] == [ref.words_of(r, 1) for r in rows]
            mask = mask_of(m, rows, [len(r) - 1 for r in rows], WINDOW, SINKS, m + k)
            for l in range(s.layers):
                q = heads_of(tables[l][tokens[b]], k, s.H, s.Hkv, s.dh)[0]
                kv = tables[l][done[b][:-1] + tokens[b], s.H * s.dh:].double().reshape(m + k, 2, s.Hkv, s.dh)
                wo, _, eo, _ = aref.forward(q, kv[:, 0], kv[:, 1], mask, TDT[dtype])
                aref.inside(outs[l][at].reshape(k, s.H, s.dh), wo, eo, f"step {step}, layer {l}, document {b}")
            width = s.H * s.dh
            want = torch.cat([o[at].double() for o in outs], 1) @ s.head.cpu().double()
            size = torch.cat([o[at].double().abs() for o in outs], 1) @ s.head.cpu().double().abs()
            aref.inside(target[at], want, 2.0 ** -23 * s.layers * width * size, f"logits of step {step}, document {b}")
            kept_rows, last = ref.walk(target[at], None, tokens[b], parents[b], u[at], v[b], temperature)
            assert path[b] == kept_rows + [-1] * (n - len(kept_rows)) and kept[b] == len(kept_rows) and token[b] == last, (step, b)
            done[b] += [tokens[b][r] for r in kept_rows[1:]] + [last]
            longest = max(longest, len(kept_rows))
            assert cached[b] == len(done[b]) - 1
        for l in range(s.layers):                                   # slots of tokens that have been decided
            for b in range(B):
                for p in range(len(done[b]) - 1):
                    got = s.c[l].data[s.c[0].table[b][p // s.page], :, :, p % s.page]
                    assert torch.equal(got, s.table[l][done[b][p], s.H * s.dh:].reshape(2, s.Hkv, s.dh)), (step, l, b, p)
    assert longest > 3                                              # drafts did stay
