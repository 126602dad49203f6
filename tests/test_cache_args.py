"""The key/value cache's entry points without a GPU: what they refuse, their
workspace sizes, and the oracle's own definitions on small cases."""
import ctypes
import os

import numpy as np
import pytest

import cache_harness as H
from oracle import cache as oc
import paper_2608_05780_amd as ev


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ev.LIB_PATH):
        pytest.skip("libevisel.so not built (run __graft_entry__.build())")
    return ev.load()


P = 1 << 20        # a stand-in for an aligned device address: never read


def view(**kw):
    """A valid view of 3 sequences, 2 kv heads, d = 64, 8 pages of 16."""
    f = dict(k=P, v=P, page_table=P, length=P, seen=P, weight=P, pos=P,
             n_pages=8, page_stride=16 * 128, token_stride=128,
             head_stride=64, n_seq=3, hkv=2, d=64, page=16, max_pages=4,
             dtype=ev.BF16)
    f.update(kw)
    return ev._CacheView(**f)


def attend(lib, v, **kw):
    a = dict(hq=4, q=P, k_new=P, v_new=P, n_tok=0, tree_ptr=P, parent=None,
             max_tree=3, max_len=64, scale=0.125, out=P, lse=None,
             accumulate=0, vote=None, decay=1.0, w_new=None, ws=P,
             ws_bytes=1 << 40)
    a.update(kw)
    return lib.evisel_tree_attention(
        ctypes.byref(v) if v is not None else None, a["hq"], a["q"],
        a["k_new"], a["v_new"], a["n_tok"], a["tree_ptr"], a["parent"],
        a["max_tree"], a["max_len"], a["scale"], a["out"], a["lse"],
        a["accumulate"], a["vote"], a["decay"], a["w_new"], a["ws"],
        a["ws_bytes"], None)


def append(lib, v, **kw):
    a = dict(k_new=P, v_new=P, n_tok=0, tok_ptr=P, accept=None, n_accept=None,
             max_new=4, w_new=None)
    a.update(kw)
    return lib.evisel_cache_append(
        ctypes.byref(v) if v is not None else None, a["k_new"], a["v_new"],
        a["n_tok"], a["tok_ptr"], a["accept"], a["n_accept"], a["max_new"],
        a["w_new"], None)


def evict(lib, v, **kw):
    a = dict(budget=32, n_sink=4, n_recent=8, max_len=32, ws=P,
             ws_bytes=1 << 40)
    a.update(kw)
    return lib.evisel_cache_evict(
        ctypes.byref(v) if v is not None else None, a["budget"], a["n_sink"],
        a["n_recent"], a["max_len"], a["ws"], a["ws_bytes"], None)


BAD_VIEWS = [
    (dict(d=96), ev.ERR_UNSUPPORTED), (dict(dtype=2), ev.ERR_UNSUPPORTED),
    (dict(page=24), ev.ERR_UNSUPPORTED), (dict(page=8), ev.ERR_UNSUPPORTED),
    (dict(page=0), ev.ERR_UNSUPPORTED),
    (dict(page=1 << 21), ev.ERR_UNSUPPORTED),
    (dict(n_seq=0), ev.ERR_INVALID_ARG), (dict(hkv=0), ev.ERR_INVALID_ARG),
    (dict(max_pages=0), ev.ERR_INVALID_ARG),
    (dict(n_pages=0), ev.ERR_INVALID_ARG),
    (dict(n_pages=1 << 31), ev.ERR_INVALID_ARG),
    (dict(max_pages=(1 << 26) + 1), ev.ERR_INVALID_ARG),
    (dict(k=None), ev.ERR_INVALID_ARG), (dict(v=None), ev.ERR_INVALID_ARG),
    (dict(page_table=None), ev.ERR_INVALID_ARG),
    (dict(length=None), ev.ERR_INVALID_ARG),
    (dict(k=P + 8), ev.ERR_INVALID_ARG), (dict(v=P + 2), ev.ERR_INVALID_ARG),
    (dict(length=P + 2), ev.ERR_INVALID_ARG),
    (dict(weight=P + 4), ev.ERR_INVALID_ARG),
    (dict(pos=P + 4), ev.ERR_INVALID_ARG),
    (dict(token_stride=132), ev.ERR_INVALID_ARG),
    (dict(head_stride=68), ev.ERR_INVALID_ARG),
    (dict(page_stride=16 * 128 + 4), ev.ERR_INVALID_ARG),
    (dict(token_stride=63), ev.ERR_INVALID_ARG),
    (dict(token_stride=(1 << 24) + 8), ev.ERR_INVALID_ARG),
    (dict(token_stride=64), ev.ERR_INVALID_ARG),     # heads on one another
    (dict(head_stride=0), ev.ERR_INVALID_ARG),
    (dict(page_stride=16 * 128 - 8), ev.ERR_INVALID_ARG),
    (dict(page_stride=-16 * 128), ev.ERR_INVALID_ARG),
    (dict(page_stride=1 << 61), ev.ERR_INVALID_ARG),
]


@pytest.mark.parametrize("i", range(len(BAD_VIEWS)))
def test_bad_views_are_refused(lib, i):
    kw, want = BAD_VIEWS[i]
    for call in (attend, append, evict):
        assert call(lib, view(**kw)) == want, kw
        assert lib.evisel_last_error()
    ref = ctypes.byref(view(**kw))
    assert lib.evisel_tree_attention_workspace(ref, 4, 3, 64, 1) == 0
    assert lib.evisel_cache_evict_workspace(ref, 8, 64) == 0


def test_valid_views(lib):
    """Calls with nothing to do (no rows, nobody over the budget) pass every
    check and launch nothing."""
    for kw in ({}, dict(head_stride=16 * 64, token_stride=64),
               dict(hkv=1, head_stride=64, token_stride=64,
                    page_stride=1024),
               dict(dtype=ev.FP32), dict(n_pages=1, page_stride=64)):
        assert attend(lib, view(**kw), max_len=0) == ev.OK
        assert append(lib, view(**kw)) == ev.OK
        assert evict(lib, view(**kw)) == ev.OK
    assert attend(lib, view(seen=None, weight=None, pos=None)) == ev.OK
    assert append(lib, view(weight=None, pos=None)) == ev.OK
    # no rows or no tokens asked for
    assert append(lib, view(), n_tok=5, max_new=0, k_new=None) == ev.OK


def test_attention_arguments(lib):
    I, W = ev.ERR_INVALID_ARG, ev.ERR_WORKSPACE
    for kw in (dict(hq=3), dict(hq=0), dict(hq=2 * 4097), dict(max_tree=0),
               dict(max_tree=65), dict(max_len=-1), dict(max_len=65),
               dict(n_tok=-1), dict(tree_ptr=None), dict(k_new=None),
               dict(v_new=None), dict(scale=0.0), dict(scale=float("nan")),
               dict(scale=1e31), dict(accumulate=1, decay=float("inf"))):
        assert attend(lib, view(), **kw) == I, kw
    assert attend(lib, view(weight=None), accumulate=1) == I
    assert attend(lib, None) == I
    for kw in (dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 8),
               dict(k_new=P + 8), dict(v_new=P + 4), dict(tree_ptr=P + 1),
               dict(parent=P + 2), dict(lse=P + 2), dict(vote=P + 1),
               dict(w_new=P + 3)):
        assert attend(lib, view(), n_tok=3, **kw) == I, kw
    need = lib.evisel_tree_attention_workspace(ctypes.byref(view()), 4, 3, 64,
                                               1)
    assert need > 0
    assert attend(lib, view(), n_tok=3, accumulate=1, ws_bytes=need - 1) == W
    assert attend(lib, view(), n_tok=3, accumulate=1, ws=None) == W
    assert attend(lib, view(), n_tok=3, accumulate=1, ws=P + 128) == W


def test_append_and_evict_arguments(lib):
    I, W = ev.ERR_INVALID_ARG, ev.ERR_WORKSPACE
    assert append(lib, view(seen=None)) == I
    for kw in (dict(n_tok=-1), dict(max_new=-1), dict(tok_ptr=None),
               dict(n_tok=3, k_new=None), dict(n_tok=3, v_new=None),
               dict(n_tok=3, k_new=P + 8), dict(n_tok=3, tok_ptr=P + 2),
               dict(n_tok=3, accept=P + 1), dict(n_tok=3, n_accept=P + 2),
               dict(n_tok=3, w_new=P + 2)):
        assert append(lib, view(), **kw) == I, kw
    for kw in (dict(seen=None), dict(weight=None), dict(pos=None)):
        assert evict(lib, view(**kw)) == I
    for kw in (dict(budget=0), dict(n_sink=-1), dict(n_recent=-1),
               dict(n_sink=20, n_recent=13), dict(max_len=65),
               dict(max_len=-1), dict(n_sink=(1 << 31) - 1,
                                      n_recent=(1 << 31) - 1)):
        assert evict(lib, view(), **kw) == I, kw
    need = lib.evisel_cache_evict_workspace(ctypes.byref(view()), 32, 64)
    assert need > 0
    assert evict(lib, view(), max_len=64, ws_bytes=need - 1) == W
    assert evict(lib, view(), max_len=64, ws=P + 16) == W
    assert evict(lib, view(), max_len=64, ws=None) == W


def test_workspace_grows_with_the_bounds(lib):
    ref = ctypes.byref(view(max_pages=4096, n_pages=1 << 14))
    ws = lib.evisel_tree_attention_workspace
    assert ws(ref, 4, 1, 0, 0) <= ws(ref, 4, 1, 60000, 0)
    assert ws(ref, 4, 1, 60000, 0) < ws(ref, 4, 1, 60000, 1)
    assert ws(ref, 4, 65, 60000, 0) == 0 and ws(ref, 3, 1, 60000, 0) == 0
    assert lib.evisel_cache_evict_workspace(ref, 0, 5) == 0


# ---------------------------------------------------------------------------
def test_binding_checks(lib):
    import torch
    t, rng = H.make(torch, (5, 20), 2, 64, "bf16", device="cpu")
    x = H.tokens(torch, rng, [2, 3], 4, 2, 64, "bf16", device="cpu")
    c = H.cache_of(ev, t)
    assert c.capacity == 32 and c.page == 16
    for name in ("length", "seen", "weight", "pos", "page_table"):
        with pytest.raises((TypeError, ValueError)):
            H.cache_of(ev, dict(t, **{name: t[name].double()}))
        with pytest.raises(ValueError):
            H.cache_of(ev, dict(t, **{name: t[name][:1]} if name !=
                                "page_table" else {name: t[name].t()}))
    with pytest.raises(ValueError):
        H.cache_of(ev, dict(t, v=t["v"].transpose(1, 2)))
    with pytest.raises(ValueError):
        H.cache_of(ev, dict(t, k=t["k"].transpose(2, 3),
                            v=t["v"].transpose(2, 3)))
    with pytest.raises(TypeError):
        H.cache_of(ev, dict(t, k=t["k"].half(), v=t["v"].half()))
    ws = torch.empty(0, dtype=torch.uint8)
    out = torch.empty_like(x["q"])
    call = lambda **kw: ev.tree_attention(
        c, **dict(dict(q=x["q"], k_new=x["k_new"], v_new=x["v_new"],
                       tree_ptr=x["tree_ptr"], out=out, workspace=ws,
                       max_tree=3, max_len=20, stream=0), **kw))
    for kw in (dict(q=x["q"].float()), dict(out=out[:4]),
               dict(k_new=x["k_new"][:4], v_new=x["v_new"][:4]),
               dict(v_new=x["v_new"][:, :1]), dict(tree_ptr=x["tree_ptr"][:2]),
               dict(tree_ptr=x["tree_ptr"].long()), dict(v_new=None),
               dict(parent=x["parent"][:3]), dict(lse=torch.zeros(5, 4)),
               dict(vote=torch.zeros(5)), dict(w_new=torch.zeros(5, 2)),
               dict(decay=1.0, vote=torch.zeros(4)),
               dict(decay=1.0, w_new=torch.zeros(2, 5)),
               dict(q=x["q"].transpose(0, 1))):
        with pytest.raises((TypeError, ValueError)):
            call(**kw)
    with pytest.raises((TypeError, ValueError)):
        ev.cache_append(c, x["k_new"], x["v_new"], x["tree_ptr"], 3,
                        accept=x["parent"][:2], stream=0)
    with pytest.raises((TypeError, ValueError)):
        ev.cache_append(c, x["k_new"], x["v_new"].float(), x["tree_ptr"], 3,
                        stream=0)


def test_oracle_chain_is_causal_attention():
    import torch
    t, rng = H.make(torch, (37,), 2, 64, "fp32", device="cpu")
    x = H.tokens(torch, rng, [5], 4, 2, 64, "fp32", device="cpu")
    c, h = H.host(t), H.host(x)
    got = oc.tree_attention(c, h["q"], h["k_new"], h["v_new"], h["tree_ptr"],
                            None, 0.125)
    rows = [oc.place(c, 0, j) for j in range(37)]
    for hd in range(4):
        k = np.stack([c["k"][p, r, hd // 2] for p, r in rows])
        v = np.stack([c["v"][p, r, hd // 2] for p, r in rows])
        k = np.concatenate([k, h["k_new"][:, hd // 2]])
        v = np.concatenate([v, h["v_new"][:, hd // 2]])
        s = h["q"][:, hd] @ k.T * 0.125
        s = np.where(np.arange(42) <= 37 + np.arange(5)[:, None], s, -np.inf)
        p = np.exp(s) / np.exp(s).sum(1, keepdims=True)
        np.testing.assert_allclose(got["out"][:, hd], p @ v, rtol=1e-12,
                                   atol=1e-13)
    np.testing.assert_allclose(
        got["mass"].sum() + got["w_new"].sum(), 4 * 5, rtol=1e-12)


def test_oracle_tree_and_eviction():
    sees = oc.ancestors(np.array([-1, 0, 0, 2, 7, 4]), 6)
    want = [[0], [0, 1], [0, 2], [0, 2, 3], [4], [4, 5]]
    for i, w in enumerate(want):
        assert np.nonzero(sees[i])[0].tolist() == w
    import torch
    t, rng = H.make(torch, (8,), 1, 64, "fp32", device="cpu", evicted=2)
    c = H.host(t)
    c["pos"][0, 0, :8] = [0, 9, 2, 3, 1, 5, 6, 7]
    c["weight"][0, 0, :8] = [0, 0, 3, np.nan, 0, 3, 4, 3]
    r = oc.evict(c, 5, 1, 1)
    # kept: slot 0 (first), 1 (last), 6 (4), then 2 and 5 (3, lowest slots)
    assert r["pos"][0, 0, :5].tolist() == [0, 9, 2, 5, 6]
    assert r["length"][0] == 5
    p = int(c["page_table"][0, 0])
    np.testing.assert_array_equal(r["k"][p, 3, 0], c["k"][p, 5, 0])
