"""Moving the rows that stay refuses a cache that is given for two layers: both would move the same rows, one after the other or at once."""
import pytest

import paper_2403_10616_amd as dp
from test_attention_refusals import A
from test_draft_refusals import EINVAL, KEEP, call

MANY = [A + 4096 * i for i in range(130)]


@pytest.mark.parametrize("caches", [(A, A), (A, A + 4096, A), (A + 4096, A, A + 8192, A), MANY[:64] + [MANY[0]], MANY + [MANY[129]], MANY[:65] + [MANY[63]]])
def test_a_cache_given_twice(caches):
    assert call("dipaco_k_cache_keep", dict(KEEP, caches=caches, n_layers=len(caches))) == EINVAL
    assert "another" in dp.last_error()
    assert call("dipaco_k_cache_keep", dict(KEEP, caches=caches, n_layers=0)) == 0
