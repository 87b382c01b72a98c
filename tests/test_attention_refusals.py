"""What the window and paged attention entry points refuse, on the host and without a GPU: nothing is enqueued."""
import pytest

import paper_2403_10616_amd as dp

A = 1 << 20            # an aligned address that no refused call may use


class Ws:
    def __init__(self, n):
        self.n = n

    def numel(self):
        return self.n

    def element_size(self):
        return 1


FWD = dict(dtype=dp.BF16, qkv=A, lengths=None, o=A, lse=A, B=2, S=64, H=4, H_kv=2, dh=64, window=16, sinks=2)
BWD = dict(FWD, d_o=A, dqkv=A, dsum=A)
APPEND = dict(dtype=dp.BF16, qkv=A, row_start=A, cache_len=A, pages=A, cache=A, T=8, B=2, H=4, H_kv=2, dh=64, n_pages=4, page_size=16, pages_per_doc=2)
PAGED = dict(APPEND, o=A, lse=A, max_new=4, window=16, sinks=2, ws=A, ws_bytes=1 << 30)


def call(name, a):
    f = getattr(dp.load(), name)
    if name.endswith("window_fwd"):
        st = f(a["dtype"], a["qkv"], a["lengths"], a["o"], a["lse"], a["B"], a["S"], a["H"], a["H_kv"], a["dh"], a["window"], a["sinks"], None)
    elif name.endswith("window_bwd"):
        st = f(a["dtype"], a["qkv"], a["lengths"], a["o"], a["d_o"], a["lse"], a["dqkv"], a["dsum"], a["B"], a["S"], a["H"], a["H_kv"], a["dh"], a["window"],
               a["sinks"], None)
    elif name.endswith("append"):
        st = f(a["dtype"], a["qkv"], a["row_start"], a["cache_len"], a["pages"], a["cache"], a["T"], a["B"], a["H"], a["H_kv"], a["dh"], a["n_pages"],
               a["page_size"], a["pages_per_doc"], None)
    else:
        st = f(a["dtype"], a["qkv"], a["row_start"], a["cache_len"], a["pages"], a["cache"], a["o"], a["lse"], a["T"], a["B"], a["max_new"], a["H"], a["H_kv"],
               a["dh"], a["n_pages"], a["page_size"], a["pages_per_doc"], a["window"], a["sinks"], a["ws"], a["ws_bytes"], None)
    return st


EINVAL, ESHAPE, EALIGN, EWORKSPACE = -1, -2, -3, -4
HEADS = [(dict(dtype=2), EINVAL), (dict(dtype=-1), EINVAL), (dict(H=0), EINVAL), (dict(H_kv=0), EINVAL), (dict(H=3), ESHAPE), (dict(dh=48), ESHAPE),
         (dict(dh=256), ESHAPE), (dict(H=1 << 15, H_kv=1 << 15), ESHAPE), (dict(qkv=None), EINVAL), (dict(qkv=A + 8), EALIGN)]
WINDOW = [(dict(window=0), EINVAL), (dict(window=-3), EINVAL), (dict(sinks=-1), EINVAL)]
PADDED = [(dict(B=0), EINVAL), (dict(S=0), EINVAL), (dict(S=-1), EINVAL), (dict(S=1 << 24), ESHAPE), (dict(B=1 << 20, S=1 << 12), ESHAPE),
          (dict(lengths=A + 4), EALIGN), (dict(o=None), EINVAL), (dict(lse=None), EINVAL), (dict(lse=A + 4), EALIGN)]
CACHE = [(dict(T=-1), EINVAL), (dict(B=0), EINVAL), (dict(n_pages=0), EINVAL), (dict(pages_per_doc=0), EINVAL), (dict(page_size=8), ESHAPE),
         (dict(page_size=48), ESHAPE), (dict(page_size=512), ESHAPE), (dict(T=1 << 24), ESHAPE), (dict(B=1 << 21), ESHAPE),
         (dict(pages_per_doc=1 << 25), ESHAPE), (dict(row_start=None), EINVAL), (dict(cache_len=None), EINVAL), (dict(pages=None), EINVAL),
         (dict(cache=None), EINVAL), (dict(cache=A + 2), EALIGN)]


@pytest.mark.parametrize("name,base,bad,status", [("dipaco_k_attention_window_fwd", FWD, *x) for x in HEADS + WINDOW + PADDED] +
                         [("dipaco_k_attention_window_bwd", BWD, *x) for x in HEADS + WINDOW + PADDED +
                          [(dict(d_o=None), EINVAL), (dict(dqkv=None), EINVAL), (dict(dsum=None), EINVAL), (dict(dqkv=A + 8), EALIGN)]] +
                         [("dipaco_k_cache_append", APPEND, *x) for x in HEADS + CACHE] +
                         [("dipaco_k_attention_paged", PAGED, *x) for x in HEADS + WINDOW + CACHE +
                          [(dict(max_new=-1), EINVAL), (dict(ws=None), EINVAL), (dict(ws_bytes=0), EWORKSPACE), (dict(o=None), EINVAL), (dict(lse=A + 4), EALIGN)]])
def test_refused(name, base, bad, status):
    assert call(name, dict(base, **bad)) == status
    assert dp.last_error()


def test_nothing_to_do_is_no_error():
    assert call("dipaco_k_cache_append", dict(APPEND, T=0, qkv=None)) == 0
    assert call("dipaco_k_attention_paged", dict(PAGED, T=0, qkv=None, ws=None, ws_bytes=0)) == 0
    assert call("dipaco_k_attention_paged", dict(PAGED, max_new=0)) == 0


def test_paged_workspace_grows_with_every_size():
    base = dict(T=64, B=4, max_new=16, H=8, H_kv=2, dh=64, page_size=16, pages_per_doc=100)

    def size(**kw):
        return dp.dipaco_k_attention_paged_workspace_bytes(*dict(base, **kw).values())

    assert size() > 0
    for name, values in dict(T=[0, 1, 64, 65, 1000, 30000], B=[1, 2, 4, 64, 1000], max_new=[0, 1, 16, 17, 100, 2000],
                             pages_per_doc=[1, 3, 10, 100, 1000, 100000], page_size=[16, 32, 64, 128, 256]).items():
        got = [size(**{name: v}) for v in values]
        assert got == sorted(got), (name, got)
    assert size(H=3) == 0 and size(dh=40) == 0 and size(page_size=5) == 0 and size(T=-1) == 0 and size(B=0) == 0 and size(max_new=-1) == 0
