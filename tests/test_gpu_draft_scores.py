"""Verification of drafts where a row's scores reach far: finite masks, rows of nothing but the lowest value, temperatures near 0."""
import pytest
import torch

import paper_2403_10616_amd as dp
from test_gpu_drafts import MODES, TYPES, check_verify
from test_gpu_window import TDT

pytestmark = pytest.mark.gpu

# Documents whose rows' sums are formed ahead of the walks: all rows', those of rows with children (documents of few rows, more than 4096 parts of a
# thousand scores), none (documents of many rows, more than 16384 parts)
AHEAD = pytest.mark.parametrize("counts", [[6, 3, 0, 9], [7, 16, 0, 12] * 8, [40, 33, 37] * 7])


def keep_top(scores, k, value):
    """all but the k largest scores of each row are `value`"""
    least = torch.topk(scores.float(), k, 1).values[:, -1:]
    scores[scores.float() < least] = value


@TYPES
@MODES
@AHEAD
@pytest.mark.parametrize("value,temperature", [("lowest", 0.7), ("lowest", 1.3), (-1e30, 1.0), ("lowest", 0.0)])
def test_scores_below_the_largest_are_masked_by_a_finite_value(dtype, mode, counts, value, temperature):
    """a few of 32000 tokens are left: whole parts of a row hold nothing but the mask's value.  The draft masks other tokens than the target"""
    value = torch.finfo(TDT[dtype]).min if value == "lowest" else value

    def special(target, draft):
        keep_top(target, 50, value)
        keep_top(draft, 40, value)

    check_verify(dtype, counts, "level", 32000, mode, temperature, draft_temperature=0.8, near=0.3, special=special, seed=21)


@TYPES
@MODES
@AHEAD
@pytest.mark.parametrize("value,temperature", [("lowest", 0.7), ("lowest", 0.8), (-1e30, 1.0), (1e20, 1.0)])
def test_rows_of_one_value(dtype, mode, counts, value, temperature):
    """all of a row's scores are the mask's value: every token is as likely as any other, of target rows, draft rows and both"""
    value = torch.finfo(TDT[dtype]).min if value == "lowest" else value

    def special(target, draft):
        target[0::3] = value
        draft[0::2] = value

    check_verify(dtype, counts, "level", 25001, mode, temperature, draft_temperature=temperature, special=special, seed=22)


@TYPES
@MODES
@pytest.mark.parametrize("temperature", [1e-5, 1e-12, 1e-20, 1e-38, 1e-45])
@pytest.mark.parametrize("V,counts", [(300, [6, 3, 20]), (32000, [6, 3]), (32000, [40, 33, 37] * 7)])
def test_temperatures_near_zero(dtype, mode, temperature, V, counts):
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
