"""Windowed and paged attention where results are not ordinary: infinities that a row sees, documents longer than their table, bits of the
probabilities, batches of more documents than one launch or one wave takes, and every check with `attention_reference.inside`, which no NaN
passes."""
import math
import random

import pytest
import torch

import attention_reference as ref
import paper_2403_10616_amd as dp
import test_gpu_paged
import test_gpu_window
from gpu_util import DEV
from test_gpu_paged import Cache, i32, starts_of
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
