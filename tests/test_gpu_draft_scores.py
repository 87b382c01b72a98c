"""Verification of drafts where a row's scores reach far: finite masks, rows of nothing but the lowest value, temperatures near 0."""
import pytest
import torch

import draft_reference as ref
import paper_2403_10616_amd as dp
from test_gpu_drafts import MODES, TYPES, check_verify, verify
from test_gpu_paged import guarded_workspace
from test_gpu_window import TDT

pytestmark = pytest.mark.gpu

# Documents whose rows' sums are formed ahead of the walks, at 32000 tokens: all rows', those of rows with children (more than 4096 parts of a thousand scores),
# none (more than 65536, without draft scores 32768)
MANY = [40, 33, 37] * 10
FEW, SOME = [6, 3, 0, 9], [7, 16, 0, 12] * 8


def keep_top(scores, k, value):
    """all but the k largest scores of each row are `value`"""
    least = torch.topk(scores.float(), k, 1).values[:, -1:]
    scores[scores.float() < least] = value


@TYPES
@MODES
@pytest.mark.parametrize("shape,temperature", [("level", 0.8), ("deep", 0.0)])
def test_many_rows_whose_sums_are_formed_in_the_walk(dtype, mode, shape, temperature):
    lengths = check_verify(dtype, MANY, shape, 32000, mode, temperature, near=0.3, seed=25)
    assert mode == "picked" or max(lengths) > 1                     # drawn drafts do stay


@TYPES
@MODES
@pytest.mark.parametrize("counts,shape", [([40] * 8, "chain"), ([40, 64, 0, 33] * 3, "deep")])
def test_long_chains_whose_sums_are_formed_ahead(dtype, mode, counts, shape):
    """more than 16 rows a document, up to 65536 parts"""
    check_verify(dtype, counts, shape, 32000, mode, 0.9, near=0.3, seed=26)


@TYPES
@MODES
@pytest.mark.parametrize("counts,value,temperature", [(FEW, "lowest", 0.7), (FEW, "lowest", 1.3), (FEW, -1e30, 1.0), (FEW, "lowest", 0.0), (SOME, "lowest", 0.7),
                                                      (SOME, -1e30, 1.0), (MANY, "lowest", 1.3), (MANY, "lowest", 0.0)])
def test_scores_below_the_largest_are_masked_by_a_finite_value(dtype, mode, counts, value, temperature):
    """a few of 32000 tokens are left: whole parts of a row hold nothing but the mask's value.  The draft masks other tokens than the target"""
    value = torch.finfo(TDT[dtype]).min if value == "lowest" else value

    def special(target, draft):
        keep_top(target, 50, value)
        keep_top(draft, 40, value)

    check_verify(dtype, counts, "level", 32000, mode, temperature, draft_temperature=0.8, near=0.3, special=special, seed=21)


@TYPES
@MODES
@pytest.mark.parametrize("counts,value,temperature", [(FEW, "lowest", 0.7), (FEW, "lowest", 0.8), (FEW, -1e30, 1.0), (FEW, 1e20, 1.0), (SOME, "lowest", 0.8),
                                                      (MANY, -1e30, 1.0)])
def test_rows_of_one_value(dtype, mode, counts, value, temperature):
    """all of a row's scores are the mask's value: every token is as likely as any other, of target rows, draft rows and both"""
    value = torch.finfo(TDT[dtype]).min if value == "lowest" else value

    def special(target, draft):
        target[0::3] = value
        draft[0::2] = value

    check_verify(dtype, counts, "level", 32000, mode, temperature, draft_temperature=temperature, special=special, seed=22)


@TYPES
@MODES
@pytest.mark.parametrize("V,counts,temperature", [(V, c, t) for t in (1e-5, 1e-12, 1e-20, 1e-38, 1e-45) for V, c in ((300, [6, 3, 20]), (32000, [6, 3]))] +
                         [(32000, [16, 9, 12] * 8, 1e-12), (32000, MANY, 1e-20)])
def test_temperatures_near_zero(dtype, mode, V, counts, temperature):
    """of the target and of the draft: all probability at the largest score, shared by those that equal it"""
    def special(target, draft):
        draft += 9.1
        target.copy_(draft.float() + 0.5 * torch.randn(draft.shape, generator=torch.Generator().manual_seed(4)))
        for x in (target, draft):
            x[1::4, 7:60:9] = 31.0                                 # several largest ones
            x[2::4] -= 40.0

    for draft_temperature in (1.0, temperature):
        check_verify(dtype, counts, "level", V, mode, temperature, draft_temperature=draft_temperature, special=special, seed=23)
    check_verify(dtype, counts, "level", V, mode, 1.0, draft_temperature=temperature, special=special, seed=24)


# documents of 65 rows in vocabularies of many parts: all rows' sums ahead, those of rows with children, none
PICKED = pytest.mark.parametrize("B,V", [(1, 60), (1, 32000), (4, 32000), (16, 32000)])


def picked(dtype, B, V, scores, tokens, u, v):
    """every document: a root with children of these tokens, each with u; its row's scores, the other rows' and tokens' far below"""
    n = len(tokens) + 1
    target = torch.full((B * n, V), -300.0)
    target[:, :len(scores)] = torch.tensor(scores)
    target = target.to(TDT[dtype])
    given = [0] + tokens
    path, kept, token = verify(dtype, target, None, given * B, [[-1] + [0] * (n - 1)] * B, torch.tensor(([0.0] + u) * B), torch.tensor(v))
    for b in range(B):
        want, last = ref.walk(target[:n], None, given, [-1] + [0] * (n - 1), torch.tensor([0.0] + u), v[b], 1.0)
        assert path[b] == want + [-1] * (n - len(want)) and kept[b] == len(want) and token[b] == last, (b, path[b], want, token[b], last)
    return kept, token


@TYPES
@PICKED
@pytest.mark.parametrize("refused", [20, 50, 64])
def test_many_picked_tokens_are_refused(dtype, B, V, refused):
    """each holds half of what the ones before it have left, down to 2^-64 of the row: what is then left decides about the next, and is what is drawn from"""
    step = 0.6875                                                   # a token's share of what is left: 1 - e^-0.6875 = 0.497
    scores = [-step * k for k in range(V if V < 100 else 200)]
    v = [(0.3, 0.7, 0.95, 0.1, 0.55, 0.8, 0.2, 0.9)[b % 8] for b in range(B)]
    tokens = [min(k, len(scores) - 1) for k in range(64)]
    kept, token = picked(dtype, B, V, scores, tokens, [0.75 if k < refused else 0.25 for k in range(64)], v)
    if refused < min(len(scores) - 4, 64):
        assert kept == [2] * B                                      # the first that is not refused is taken
    if refused == 64 and V > 100:
        assert min(token) >= 64


@TYPES
@PICKED
def test_picked_tokens_of_almost_all_probability_are_refused(dtype, B, V):
    """random numbers just below 1: of the row 1e-7, 1e-14 and 1e-21 are left"""
    top = 1 - 2.0 ** -24
    for u, want in (([top, top, top, 0.5], [0, 4]), ([top, top, top, top], None)):
        kept, token = picked(dtype, B, V, [0.0, -16.0, -32.0, -48.0, -64.0, -64.0], [0, 1, 2, 3] + [-1] * 60, u + [0.0] * 60, [0.75] * B)
        assert kept == [2 if want else 1] * B and (want or token == [5] * B)


@pytest.mark.parametrize("draft,rows", [(True, 32), (False, 33), (False, 32)])
def test_the_workspace_of_many_parts_is_as_large_as_it_is_said_to_be(draft, rows):
    """65536 parts of rows with draft scores, the most that are formed ahead, and a few more and a few less than the most without"""
    B, V, g = 32, 32000, torch.Generator().manual_seed(5)
    T = B * rows
    target = 8 * torch.randn(T, V, generator=g)
    scores = target + 0.3 * torch.randn(T, V, generator=g) if draft else None
    args = (dp.F32, target, scores, target.argmax(1).roll(1).tolist(), [list(range(-1, rows - 1))] * B, torch.rand(T, generator=g), torch.rand(B, generator=g))
    n = dp.dipaco_k_draft_verify_workspace_bytes(T, B, V)
    whole, ws = guarded_workspace(n)
    got = verify(*args, ws=ws)
    assert got == verify(*args) and max(got[1]) > 2
    assert bool((whole[:4096] == 170).all()) and bool((whole[4096 + n:] == 170).all())
