"""What the entry points of drafted decoding refuse, on the host and without a GPU: nothing is enqueued."""
import ctypes as C

import pytest

import paper_2403_10616_amd as dp
from test_attention_refusals import A, CACHE, HEADS, WINDOW

EINVAL, ESHAPE, EALIGN, EWORKSPACE = -1, -2, -3, -4
TREE = dict(parent=A, row_start=A, depth=A, seen=A, T=8, B=2, max_new=4)
ATTEND = dict(dtype=dp.BF16, qkv=A, row_start=A, cache_len=A, depth=A, seen=A, pages=A, cache=A, o=A, lse=A, T=8, B=2, max_new=4, H=4, H_kv=2, dh=64,
              n_pages=4, page_size=16, pages_per_doc=2, window=16, sinks=2, ws=A, ws_bytes=1 << 30)
VERIFY = dict(dtype=dp.BF16, target=A, draft=A, tokens=A, parent=A, row_start=A, u=A, v=A, path=A, kept=A, next=A, T=8, B=2, max_new=4, V=100,
              temperature=1.0, draft_temperature=1.0, distinct=0, ws=A, ws_bytes=1 << 20)
KEEP = dict(dtype=dp.BF16, path=A, kept=A, cache_len=A, pages=A, caches=(A, A), n_layers=2, B=2, max_new=4, H_kv=2, dh=64, n_pages=4, page_size=16,
            pages_per_doc=2)


def call(name, a):
    a = dict(a)
    if a.get("caches") is not None:
        a["caches"] = (C.c_void_p * len(a["caches"]))(*a["caches"])
    return getattr(dp.load(), name)(*a.values(), None)


DRAFTS = [(dict(T=-1), EINVAL), (dict(B=0), EINVAL), (dict(max_new=-1), EINVAL), (dict(max_new=1025), ESHAPE), (dict(T=1 << 24), ESHAPE), (dict(B=1 << 21), ESHAPE)]
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("name,base,bad,status", [("dipaco_k_draft_tree", TREE, *x) for x in DRAFTS +
                          [(dict(parent=None), EINVAL), (dict(row_start=None), EINVAL), (dict(depth=None), EINVAL), (dict(seen=None), EINVAL),
                           (dict(seen=A + 8), EALIGN)]] +
                         [("dipaco_k_attention_tree", ATTEND, *x) for x in HEADS + WINDOW + CACHE + DRAFTS +
                          [(dict(window=3), ESHAPE), (dict(depth=None), EINVAL), (dict(seen=None), EINVAL), (dict(seen=A + 8), EALIGN), (dict(ws=None), EINVAL),
                           (dict(ws_bytes=0), EWORKSPACE), (dict(o=None), EINVAL), (dict(lse=A + 4), EALIGN)]] +
                         [("dipaco_k_draft_verify", VERIFY, *x) for x in DRAFTS +
                          [(dict(dtype=2), EINVAL), (dict(V=0), EINVAL), (dict(V=(1 << 18) + 1), ESHAPE), (dict(temperature=-1.0), EINVAL),
                           (dict(temperature=INF), EINVAL), (dict(temperature=NAN), EINVAL), (dict(draft_temperature=0.0), EINVAL),
                           (dict(draft_temperature=-1.0), EINVAL), (dict(draft_temperature=NAN), EINVAL), (dict(distinct=2), EINVAL),
                           (dict(ws_bytes=8), EWORKSPACE), (dict(draft=A + 2), EALIGN)] +
                          [({k: None}, EINVAL) for k in ("target", "tokens", "parent", "row_start", "u", "v", "path", "kept", "next", "ws")]] +
                         [("dipaco_k_cache_keep", KEEP, *x) for x in
                          [(dict(dtype=2), EINVAL), (dict(H_kv=0), EINVAL), (dict(dh=48), ESHAPE), (dict(n_layers=-1), EINVAL), (dict(B=0), EINVAL),
                           (dict(max_new=-1), EINVAL), (dict(max_new=2000), ESHAPE), (dict(n_pages=0), EINVAL), (dict(page_size=24), ESHAPE),
                           (dict(pages_per_doc=0), EINVAL), (dict(path=None), EINVAL), (dict(kept=None), EINVAL), (dict(cache_len=None), EINVAL),
                           (dict(pages=None), EINVAL), (dict(caches=None), EINVAL), (dict(caches=(A, 0)), EINVAL), (dict(caches=(A, A + 8)), EALIGN)]])
def test_refused(name, base, bad, status):
    assert call(name, dict(base, **bad)) == status
    assert dp.last_error()


def test_nothing_to_do_is_no_error():
    assert call("dipaco_k_draft_tree", dict(TREE, T=0, parent=None, depth=None, seen=None)) == 0
    assert call("dipaco_k_attention_tree", dict(ATTEND, T=0, qkv=None, ws=None, ws_bytes=0)) == 0
    assert call("dipaco_k_attention_tree", dict(ATTEND, max_new=0)) == 0
    assert call("dipaco_k_cache_keep", dict(KEEP, n_layers=0, caches=None)) == 0
    assert call("dipaco_k_cache_keep", dict(KEEP, max_new=0)) == 0


def test_workspaces_grow_with_every_size():
    base = dict(T=64, B=4, max_new=16, H=8, H_kv=2, dh=64, page_size=16, pages_per_doc=100)

    def size(**kw):
        return dp.dipaco_k_attention_tree_workspace_bytes(*dict(base, **kw).values())

    assert size() > 0
    for name, values in dict(T=[0, 1, 64, 65, 1000, 30000], B=[1, 2, 4, 64, 1000], max_new=[0, 1, 16, 17, 100, 1024],
                             pages_per_doc=[1, 3, 10, 100, 1000, 100000], page_size=[16, 32, 64, 128, 256]).items():
        got = [size(**{name: v}) for v in values]
        assert got == sorted(got), (name, got)
    assert size(H=3) == 0 and size(dh=40) == 0 and size(page_size=5) == 0 and size(T=-1) == 0 and size(B=0) == 0 and size(max_new=1025) == 0
    base = dict(T=64, B=4, V=1000)
    for name, values in dict(T=[0, 1, 64, 1000, 1 << 23], B=[1, 2, 100, 1 << 20], V=[1, 2, 1001, 32000, 1 << 18]).items():
        got = [dp.dipaco_k_draft_verify_workspace_bytes(*dict(base, **{name: v}).values()) for v in values]
        assert got == sorted(got) and got[0] > 0, (name, got)
    for bad in (dict(T=-1), dict(B=0), dict(V=0), dict(V=(1 << 18) + 1)):
        assert dp.dipaco_k_draft_verify_workspace_bytes(*dict(base, **bad).values()) == 0
