"""The key/value cache on the GPU against the fp64 oracle: attention of drafted
trees over paged caches, accumulated weights, append and eviction, and the
three used together. The bounds are tolerances() of the harness, from the
number formats alone."""
import numpy as np
import pytest

import cache_harness as H
from gpu_harness import say
from oracle import cache as oc

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _lib(gpu_lib):
    pytest.ev = gpu_lib


def attend(t, x, max_tree=None, max_len=None, decay=None, vote=None,
           chain=False, scale=None, alone=False, ws=None, stream=None,
           filled=3.0):
    """Runs the call; outputs as fp64 arrays (out, lse, weight, w_new)."""
    import torch
    ev = pytest.ev
    c = H.cache_of(ev, t)
    n_tok, hq, d = x["q"].shape
    ns = x["tree_ptr"].diff()
    mt = max_tree or max(1, int(ns.max()))
    ml = c.capacity if max_len is None else max_len
    out = torch.full_like(x["q"], filled)
    lse = torch.full((hq, n_tok), filled, device="cuda")
    wn = torch.full((n_tok, c.hkv), filled, device="cuda")
    need = ev.tree_attention_workspace(c, hq, mt, ml, decay is not None)
    if ws is None:   # poisoned: nothing may be read that was not written
        ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()   # the call may be on another stream
    ev.tree_attention(c, x["q"], None if alone else x["k_new"],
                      None if alone else x["v_new"], x["tree_ptr"], out, ws,
                      max_tree=mt, max_len=ml,
                      parent=None if chain else x["parent"], lse=lse,
                      vote=vote, decay=decay,
                      w_new=None if decay is None else wn,
                      softmax_scale=scale, stream=stream)
    torch.cuda.synchronize()
    return H.host({"out": out, "lse": lse, "weight": t["weight"],
                   "w_new": wn})


def check(t, x, dtype, max_tree=None, max_len=None, decay=None, vote=None,
          chain=False, scale=None, alone=False, **kw):
    before = H.host(t)
    h = H.host(x)
    d = h["q"].shape[2]
    scale = scale or d ** -0.5
    ref = oc.tree_attention(
        before, h["q"], None if alone else h["k_new"],
        None if alone else h["v_new"], h["tree_ptr"],
        None if chain else h["parent"], scale,
        vote=None if vote is None else vote.cpu().double().numpy(),
        decay=1.0 if decay is None else decay, max_tree=max_tree or 64,
        max_len=max_len)
    got = attend(t, x, max_tree, max_len, decay, vote, chain, scale, alone,
                 **kw)
    ns = np.diff(h["tree_ptr"])
    keys = int(before["length"].max()) + int(ns.max())
    tol = H.tolerances(ref, d, dtype, keys, int(ns.max()) * h["q"].shape[1],
                       1.0 if decay is None else decay, before["weight"])
    live = np.zeros(h["q"].shape[0], bool)
    for a, n in zip(h["tree_ptr"], ns):
        live[a:a + min(n, max_tree or 64)] = True
    H.close("out", got["out"][live], ref["out"][live], tol["out"][live])
    H.close("lse", got["lse"][:, live], ref["lse"][:, live],
            tol["lse"][:, live])
    # rows outside the sequences: as they were
    assert (got["out"][~live] == 3.0).all() and (got["lse"][:, ~live] == 3.0).all()
    if decay is None:
        assert np.array_equal(got["weight"], before["weight"])
        assert (got["w_new"] == 3.0).all()
    else:
        H.close("weight", got["weight"], ref["weight"], tol["weight"])
        H.close("w_new", got["w_new"][live], ref["w_new"][live],
                tol["w_new"][live])
        assert (got["w_new"][~live] == 3.0).all()
    return got


MODELS = {"bf16-7": (28, 4, 128, "bf16"), "bf16-d64": (12, 2, 64, "bf16"),
          "fp32-d64": (4, 1, 64, "fp32"), "fp32-7": (14, 2, 128, "fp32"),
          "mha": (3, 3, 128, "bf16"), "mqa": (20, 1, 64, "bf16")}


@pytest.mark.parametrize("model", list(MODELS))
@pytest.mark.parametrize("lens", [(1,), (0, 15, 16, 17), (31, 32, 33),
                                  (63, 64, 65, 700), (2049, 130, 1)])
def test_one_token(model, lens):
    import torch
    hq, hkv, d, dt = MODELS[model]
    t, rng = H.make(torch, lens, hkv, d, dt, page=16, seed=len(lens))
    x = H.tokens(torch, rng, [1] * len(lens), hq, hkv, d, dt)
    say(f"  one token {model} {lens}")
    check(t, x, dt)
    check(t, x, dt, decay=0.75)


@pytest.mark.parametrize("model", list(MODELS))
@pytest.mark.parametrize("ns", [(2, 0, 5), (17, 1, 33), (64, 0, 31)])
def test_trees(model, ns):
    import torch
    hq, hkv, d, dt = MODELS[model]
    t, rng = H.make(torch, (260, 77, 0), hkv, d, dt, page=32, seed=sum(ns),
                    layout="head")
    x = H.tokens(torch, rng, list(ns), hq, hkv, d, dt, slack=3)
    vote = torch.rand(x["q"].shape[0], device="cuda")
    vote[0] = 0.0
    say(f"  trees {model} {ns}")
    check(t, x, dt)
    check(t, x, dt, decay=1.0, vote=vote)
    check(t, x, dt, chain=True, decay=0.0)


@pytest.mark.parametrize("page,layout", [(16, "wide"), (32, "token"),
                                         (64, "head"), (256, "wide"),
                                         (4096, "token")])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_pages_and_strides(page, layout, dt):
    import torch
    t, rng = H.make(torch, (1000, 33), 2, 128, dt, page=page, layout=layout)
    x = H.tokens(torch, rng, [3, 20], 6, 2, 128, dt)
    say(f"  pages of {page} {layout} {dt}")
    check(t, x, dt, decay=0.5)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_cache_alone(dt):
    """Without new keys: the cache holds what the tokens see. An empty cache
    leaves a row without keys: zeros, lse -inf, no weight."""
    import torch
    t, rng = H.make(torch, (40, 0, 129), 2, 64, dt)
    x = H.tokens(torch, rng, [1, 2, 30], 4, 2, 64, dt)
    got = check(t, x, dt, alone=True, decay=1.0)
    assert (got["out"][1:3] == 0).all() and np.isneginf(got["lse"][:, 1:3]).all()
    assert (got["w_new"] == 0).all()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_steep_rows(dt):
    """Logits in the hundreds, growing along the cache: the reference moves
    all the way; and the other way round."""
    import torch
    for flip in (False, True):
        t, rng = H.make(torch, (900,), 1, 64, dt, page=1024)
        ramp = torch.linspace(0, 12, 1024, device="cuda")
        if flip:
            ramp = ramp.flip(0)
        page = int(t["page_table"][0, 0])
        t["k"][page] *= 0.05
        t["k"][page, :, 0, 0] = ramp.to(t["k"].dtype)
        x = H.tokens(torch, rng, [2], 2, 1, 64, dt)
        x["q"][:, :, 0] = 200.0
        check(t, x, dt, decay=1.0)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("n", [1, 9])
def test_rows_of_minus_infinity(dt, n):
    """Every key's logit is -inf: zeros, lse -inf, and no weight."""
    import torch
    t, rng = H.make(torch, (70,), 1, 64, dt)
    x = H.tokens(torch, rng, [n], 2, 1, 64, dt)
    x["q"].zero_()
    x["q"][:, :, 3] = 1.0
    t["k"][..., 3] = float("-inf")
    x["k_new"][..., 3] = float("-inf")
    got = check(t, x, dt, decay=1.0)
    assert (got["out"] == 0).all() and np.isneginf(got["lse"]).all()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("hq", [2, 20])
def test_values_that_are_not_finite(dt, bad, hq):
    """In a drafted token's key or value, they reach the rows that see the
    token and no other; past a sequence's length, and in rows of the pool that
    belong to nobody, they reach nothing."""
    import torch
    for which in ("k_new", "v_new"):
        t, rng = H.make(torch, (70, 16, 0), 1, 64, dt)
        for s, ln in enumerate((70, 16, 0)):
            p = int(t["page_table"][s, (ln - 1) // 16]) if ln else 0
            if ln % 16:
                t["k"][p, ln % 16:] = bad
                t["v"][p, ln % 16:] = bad
        x = H.tokens(torch, rng, [6, 40, 3], hq, 1, 64, dt)
        # token 2 of the first tree, 35 of the second; leaves and inner ones
        x["parent"][:6] = torch.tensor([-1, 0, 0, 2, 1, 3])
        x[which][2, :, 5] = bad
        x[which][6 + 35, :, 5:9] = bad
        got = check(t, x, dt)
        assert np.isfinite(got["out"][[0, 1, 4]]).all()
        assert not np.isfinite(got["out"][[2, 3, 5]]).all()


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_pages_that_are_not_there(dt):
    """Table entries outside the pool hold nothing (and nothing is read)."""
    import torch
    t, rng = H.make(torch, (200, 64), 2, 64, dt, page=16)
    t["page_table"][0, 0] = -1
    t["page_table"][0, 5] = 1 << 30
    t["page_table"][1, :] = t["k"].shape[0]
    x = H.tokens(torch, rng, [2, 2], 4, 2, 64, dt)
    check(t, x, dt)
    check(t, x, dt, decay=0.5)
    x = H.tokens(torch, rng, [20, 9], 4, 2, 64, dt)
    check(t, x, dt, decay=0.5)


def test_parents_that_are_none():
    """A parent that is the token itself, a later one or far away: a root."""
    import torch
    t, rng = H.make(torch, (50,), 1, 64, "bf16")
    x = H.tokens(torch, rng, [6], 2, 1, 64, "bf16")
    x["parent"][:] = torch.tensor([0, 1, 5, -7, 1 << 30, 2])
    check(t, x, "bf16", decay=1.0)


def test_bounds_leave_the_rest_out():
    """max_tree and max_len below what the device arrays say."""
    import torch
    t, rng = H.make(torch, (300, 90), 2, 128, "bf16", page=16)
    x = H.tokens(torch, rng, [12, 3], 8, 2, 128, "bf16")
    check(t, x, "bf16", max_tree=5, max_len=100, decay=1.0)
    check(t, x, "bf16", max_tree=2, max_len=0, decay=1.0)
    check(t, x, "bf16", max_tree=1, max_len=17, decay=1.0)


def test_more_splits_than_work_and_fewer():
    """Long and short sequences in one call, with the bound at the capacity."""
    import torch
    t, rng = H.make(torch, (9000, 1, 33), 1, 128, "bf16", page=64)
    x = H.tokens(torch, rng, [1, 1, 1], 8, 1, 128, "bf16")
    check(t, x, "bf16", decay=1.0)
    t, rng = H.make(torch, (5000,), 4, 128, "bf16", page=64)
    x = H.tokens(torch, rng, [64], 28, 4, 128, "bf16", scale=2.0)
    check(t, x, "bf16")


def test_loose_bound():
    """A bound of 2^25 tokens on a cache of 300: the workspace stays within 1
    GiB for the logits of 16 rows, and the weights are the same."""
    import torch
    ev = pytest.ev
    t, rng = H.make(torch, (300,), 1, 64, "bf16", page=64)
    cap = 1 << 25
    table = torch.full((1, cap // 64), -1, dtype=torch.int32, device="cuda")
    table[:, :t["page_table"].shape[1]] = t["page_table"]
    old = t["weight"].shape[2]
    t.update(page_table=table, pos=None)
    w = torch.zeros(1, 1, cap, device="cuda")
    w[:, :, :old] = t["weight"]
    t["weight"] = w
    x = H.tokens(torch, rng, [2], 8, 1, 64, "bf16")
    assert ev.tree_attention_workspace(H.cache_of(ev, t), 8, 2, cap,
                                       True) < 1 << 30
    check(t, x, "bf16", decay=0.5)


def test_offsets_past_32_bits():
    """Pages more than 2^32 bytes from the pool's start."""
    import torch
    far = (1 << 28) + 64                       # elements between pages
    for dt in (torch.bfloat16, torch.float32):
        t, rng = H.make(torch, (150,), 2, 64,
                        "bf16" if dt == torch.bfloat16 else "fp32", page=16,
                        extra=20, evicted=3)
        n_pages = t["k"].shape[0]
        for name in ("k", "v"):
            pool = torch.empty(far * n_pages, dtype=dt, device="cuda")
            p = pool.as_strided(t[name].shape, (far, 2 * 64, 64, 1))
            p.copy_(t[name])
            t[name] = p
        x = H.tokens(torch, rng, [3], 4, 2, 64,
                     "bf16" if dt == torch.bfloat16 else "fp32")
        say(f"  offsets up to {far * n_pages * t['k'].element_size() >> 30} GiB")
        name = "bf16" if dt == torch.bfloat16 else "fp32"
        check(t, x, name, decay=1.0)
        run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], 64)
        run_evict(t, 100, 4, 20)
        del t, p, pool
        torch.cuda.empty_cache()


# ---------------------------------------------------------------------------
def same(t, want):
    got = H.host(t)
    for name in want:
        assert np.array_equal(got[name], want[name], equal_nan=True), name


def run_append(t, k_new, v_new, ptr, max_new, **kw):
    import torch
    ev = pytest.ev
    h = {k: None if v is None else v.cpu().double().numpy()
         if v.is_floating_point() else v.cpu().numpy() for k, v in kw.items()}
    want = oc.append(H.host(t), k_new.cpu().double().numpy(),
                     v_new.cpu().double().numpy(), ptr.cpu().numpy(), max_new,
                     **h)
    ev.cache_append(H.cache_of(ev, t), k_new, v_new, ptr, max_new, **kw)
    torch.cuda.synchronize()
    same(t, want)


@pytest.mark.parametrize("model", list(MODELS))
@pytest.mark.parametrize("ns", [(1, 0, 7), (64, 3, 20), (700, 0, 90)])
def test_append(model, ns):
    import torch
    hq, hkv, d, dt = MODELS[model]
    t, rng = H.make(torch, (0, 31, 100), hkv, d, dt, extra=max(ns), evicted=9)
    x = H.tokens(torch, rng, list(ns), hq, hkv, d, dt, slack=2)
    w = torch.rand(x["q"].shape[0], hkv, device="cuda")
    say(f"  append {model} {ns}")
    run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], max(ns), w_new=w)
    t, rng = H.make(torch, (5, 0, 64), hkv, d, dt, extra=max(ns),
                    layout="head", page=64)
    run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], max(ns))


def test_append_picks():
    """Accepted paths: counts past the rows, indices outside them, the same
    index twice, a bound below the counts, and no room."""
    import torch
    t, rng = H.make(torch, (40, 10, 0, 31), 2, 64, "bf16", extra=8)
    x = H.tokens(torch, rng, [9, 4, 0, 5], 4, 2, 64, "bf16")
    n = x["q"].shape[0]
    acc = torch.from_numpy(rng.integers(0, 4, n).astype(np.int32)).cuda()
    acc[1], acc[2] = 1 << 30, -3
    for cnt, bound in (([3, 4, 0, 1], 9), ([100, -2, 5, 5], 9),
                       ([9, 4, 0, 5], 2)):
        run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], bound,
                   accept=acc,
                   n_accept=torch.tensor(cnt, dtype=torch.int32, device="cuda"))
    # the capacity: what does not fit is left out and not counted
    for _ in range(3):
        run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], 9)
    assert int(t["length"].max()) == t["weight"].shape[2]


def test_append_many_past_the_capacity():
    import torch
    t, rng = H.make(torch, (700, 3), 4, 128, "bf16", page=16)
    x = H.tokens(torch, rng, [600, 300], 4, 4, 128, "bf16")
    t["page_table"][1, 10] = -1
    run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], 600)


def run_evict(t, budget, n_sink, n_recent, max_len=None):
    import torch
    ev = pytest.ev
    c = H.cache_of(ev, t)
    want = oc.evict(H.host(t), budget, n_sink, n_recent, max_len)
    ml = c.capacity if max_len is None else max_len
    ws = torch.full((ev.cache_evict_workspace(c, budget, ml) + 256,), 0xFF,
                    dtype=torch.uint8, device="cuda")
    ev.cache_evict(c, budget, ws, n_sink, n_recent, max_len)
    torch.cuda.synchronize()
    same(t, want)


@pytest.mark.parametrize("model", list(MODELS))
@pytest.mark.parametrize("lens,budget,sink,recent", [
    ((1, 2, 3), 1, 0, 0), ((1, 2, 3), 2, 1, 1), ((65, 64, 200, 0), 64, 4, 10),
    ((1100, 1025, 17), 1024, 4, 512), ((2500, 900), 333, 0, 333),
    ((500,), 499, 499, 0)])
def test_evict(model, lens, budget, sink, recent):
    import torch
    hq, hkv, d, dt = MODELS[model]
    for layout, page in (("token", 16), ("head", 64)):
        t, rng = H.make(torch, lens, hkv, d, dt, page=page, layout=layout,
                        evicted=7, seed=budget)
        say(f"  evict {model} {lens} to {budget} {layout}")
        run_evict(t, budget, sink, recent)


def test_evict_long():
    """Longer than the keys that stay in LDS."""
    import torch
    t, rng = H.make(torch, (36865, 40000, 36864), 1, 64, "bf16", page=64,
                    evicted=100)
    run_evict(t, 9000, 4, 1000)


@pytest.mark.parametrize("n", [300, 9001, 37000])
@pytest.mark.parametrize("what", ["equal", "zeros", "two", "odd", "tiny"])
def test_evict_ranks(what, n):
    """Ties to the lowest slot; NaN like -inf, -0 like 0, infinities,
    negatives and denormals in order."""
    import torch
    t, rng = H.make(torch, (n,), 2, 64, "bf16", page=64)
    w = t["weight"]
    if what == "equal":
        w.fill_(0.5)
    elif what == "zeros":
        w.zero_()
        w[:, :, ::3] = -0.0
    elif what == "two":
        w[:] = torch.where(w > 1, 2.0, 1.0)
    elif what == "tiny":
        w[:] = torch.randint(0, 50, w.shape, device="cuda") * 2.0 ** -149
    else:
        w[:, :, ::5] = float("nan")
        w[:, :, 1::7] = float("-inf")
        w[:, :, 2::11] = float("inf")
        w[:, :, 3::4] *= -1
    for budget in (n - 1, n // 2, n // 9, 1):
        u = {k: v.clone() for k, v in t.items()}
        run_evict(u, budget, 0, 0)
        if budget > 40:
            u = {k: v.clone() for k, v in t.items()}
            run_evict(u, budget, 10, 30)


def test_evict_bounds():
    """A max_len below a length takes the sequence for one of max_len; pages
    that are not there drop their moves; a budget that nobody passes changes
    nothing."""
    import torch
    t, rng = H.make(torch, (300, 100), 2, 64, "bf16")
    u = {k: v.clone() for k, v in t.items()}
    run_evict(u, 80, 4, 10, max_len=200)
    u = {k: v.clone() for k, v in t.items()}
    u["page_table"][0, 2] = -1
    u["page_table"][0, 15] = 1 << 30
    run_evict(u, 150, 4, 10)
    run_evict(t, 300, 4, 10)
    run_evict(t, 90, 4, 10, max_len=90)


# ---------------------------------------------------------------------------
def test_generation_together():
    """A cache as a program uses it: prefilled tokens in, then rounds of
    drafted trees, of which paths are accepted, and evictions; every call
    against the oracle on the state that the calls before left."""
    import torch
    ev = pytest.ev
    hq, hkv, d, dt = 14, 2, 128, "bf16"
    lens = (150, 77, 0)
    t, rng = H.make(torch, (0, 0, 0), hkv, d, dt, page=16, extra=256)
    x = H.tokens(torch, rng, list(lens), hq, hkv, d, dt)
    w0 = torch.rand(sum(lens), hkv, device="cuda")
    run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], 150, w_new=w0)
    for step in range(6):
        ns = [int(n) for n in rng.integers(0, 20, 3)]
        ns[step % 3] = max(1, ns[step % 3])
        x = H.tokens(torch, rng, ns, hq, hkv, d, dt)
        got = check(t, x, dt, decay=0.9)
        acc = np.zeros(sum(ns), np.int32)
        cnt = []
        for a, n in zip(np.concatenate([[0], np.cumsum(ns)]), ns):
            path = sorted(rng.permutation(n)[:int(rng.integers(0, n + 1))])
            acc[a:a + len(path)] = path
            cnt.append(len(path))
        wn = torch.from_numpy(got["w_new"].astype(np.float32)).cuda()
        run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], 20,
                   accept=torch.from_numpy(acc).cuda(),
                   n_accept=torch.tensor(cnt, dtype=torch.int32, device="cuda"),
                   w_new=wn)
        run_evict(t, 96, 4, 16)
    assert int(t["length"].max()) == 96


def test_after_the_probe():
    """The probe's own path and on from it: a prefilled video (all-causal
    rule) enters the cache with its evidence as first weights, and its last
    query token, attended over the cache, gets what the prefill gave it; then
    the cache is cut by those weights and the frames that held the evidence
    are still there."""
    import torch
    ev = pytest.ev
    frames, text, nv, hq, hkv, d = 20, 9, 16, 8, 2, 128
    S = frames * nv + text
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    q, k, v = rnd(S, hq, d), rnd(S, hkv, d), rnd(S, hkv, d)
    # the query tokens look at frames 6 and 13
    way = rnd(hkv, d)
    for f in (6, 13):
        k[f * nv:(f + 1) * nv] += 0.7 * way
    q[frames * nv:] += 0.7 * way.repeat_interleave(hq // hkv, 0)
    q, k, v = (x.to(torch.bfloat16) for x in (q, k, v))
    mask = ev.build_block_mask([frames], [text], nv, 64, 1, -1, hq, hkv)
    out = torch.empty_like(q)
    lse = torch.empty(hq, S, device="cuda")
    evid = torch.empty(1, hq, frames, device="cuda")
    ws = torch.empty(ev.sparse_prefill_workspace(mask, d), dtype=torch.uint8,
                     device="cuda")
    ev.sparse_prefill(mask, 0, 1, q, k, v, out, evid, ws, lse=lse)
    t, _ = H.make(torch, (0,), hkv, d, "bf16", page=16, extra=S)
    w0 = torch.zeros(S, hkv, device="cuda")
    per_kv = evid[0].view(hkv, hq // hkv, frames).sum(1) / nv
    w0[:frames * nv] = per_kv.t().repeat_interleave(nv, 0)
    ptr = torch.tensor([0, S - 1], dtype=torch.int32, device="cuda")
    run_append(t, k, v, ptr, S, w_new=w0)
    x = {"q": q[-1:].contiguous(), "k_new": k[-1:].contiguous(),
         "v_new": v[-1:].contiguous(),
         "tree_ptr": torch.tensor([0, 1], dtype=torch.int32, device="cuda"),
         "parent": torch.tensor([-1], dtype=torch.int32, device="cuda")}
    got = check(t, x, "bf16", decay=1.0)
    # both round the probabilities and the output to bf16
    h = H.host({"out": out[-1:], "lse": lse[:, -1:]})
    ref = oc.tree_attention(H.host(t), *(H.host(x)[n] for n in (
        "q", "k_new", "v_new", "tree_ptr", "parent")), d ** -0.5)
    bound = 2 * 2.0 ** -8 * (ref["absv"] + np.abs(ref["out"])) * 1.01
    assert (np.abs(h["out"] - got["out"]) <= bound).all()
    assert np.abs(h["lse"] - got["lse"]).max() <= 1e-5
    run_evict(t, 64, 2, 9)
    pos = t["pos"][0, :, :64].cpu().numpy()
    for g in range(hkv):
        kept = set(pos[g].tolist())
        for f in (6, 13):
            assert kept >= set(range(f * nv, (f + 1) * nv))


def test_results_do_not_depend_on_the_run():
    """The same call again, with another workspace: the same bits."""
    import torch
    for ns in ((1, 1), (30, 64)):
        t, rng = H.make(torch, (3000, 500), 4, 128, "bf16", page=64)
        x = H.tokens(torch, rng, list(ns), 28, 4, 128, "bf16")
        w0 = t["weight"].clone()
        a = attend(t, x, decay=0.5)
        t["weight"].copy_(w0)
        b = attend(t, x, decay=0.5)
        for k in a:
            assert np.array_equal(a[k], b[k]), k


@pytest.mark.parametrize("n_seq", [70, 300])
def test_many_sequences(n_seq):
    """More sequences than lanes, and than those whose lengths every work-group
    looks through; idle ones among them."""
    import torch
    rng = np.random.default_rng(n_seq)
    lens = tuple(int(x) for x in rng.integers(0, 200, n_seq))
    lens = lens[:-2] + (700, 0)
    ns = [int(x) for x in rng.integers(0, 6, n_seq)]
    ns[3], ns[-1] = 14, 3
    say(f"  {n_seq} sequences")
    t, r = H.make(torch, lens, 1, 64, "bf16", page=32)
    x = H.tokens(torch, r, ns, 6, 1, 64, "bf16")
    check(t, x, "bf16", decay=0.5)
    x = H.tokens(torch, r, [min(n, 1) for n in ns], 6, 1, 64, "bf16")
    check(t, x, "bf16", decay=0.5)
    run_append(t, x["k_new"], x["v_new"], x["tree_ptr"], 1)
    run_evict(t, 60, 4, 8)


def test_long_runs_and_row_blocks():
    """Many rows over a long cache next to a short one: several runs, two
    blocks of rows, the second one's keys halved."""
    import torch
    t, rng = H.make(torch, (6000, 90, 0), 1, 128, "bf16", page=64)
    x = H.tokens(torch, rng, [50, 9, 64], 7, 1, 128, "bf16")
    check(t, x, "bf16", decay=1.0)
    t["page_table"][0, 40] = -1
    t["page_table"][0, 93] = 1 << 20
    check(t, x, "bf16")


def test_two_calls_at_once():
    """Two caches on two streams with workspaces of their own: what each call
    gives alone."""
    import torch
    both = []
    for seed in (1, 2):
        t, rng = H.make(torch, (3000, 400), 2, 128, "bf16", page=64, seed=seed)
        x = H.tokens(torch, rng, [20, 3], 14, 2, 128, "bf16")
        w0 = t["weight"].clone()
        alone = attend(t, x, decay=1.0)
        t["weight"].copy_(w0)
        both.append((t, x, alone, torch.cuda.Stream()))
    ev = pytest.ev
    outs = []
    torch.cuda.synchronize()
    for t, x, _, s in both:
        c = H.cache_of(ev, t)
        with torch.cuda.stream(s):
            out = torch.empty_like(x["q"])
            lse = torch.empty(14, x["q"].shape[0], device="cuda")
            ws = torch.empty(ev.tree_attention_workspace(
                c, 14, 20, c.capacity, True), dtype=torch.uint8, device="cuda")
            ev.tree_attention(c, x["q"], x["k_new"], x["v_new"],
                              x["tree_ptr"], out, ws, 20, c.capacity,
                              parent=x["parent"], lse=lse, decay=1.0)
            outs.append((out, lse, ws))
    torch.cuda.synchronize()
    for (t, _, alone, _), (out, lse, _) in zip(both, outs):
        got = H.host({"out": out, "lse": lse, "weight": t["weight"]})
        for k in got:
            assert np.array_equal(got[k], alone[k]), k


def test_host_memory_is_refused():
    import torch
    ev = pytest.ev
    t, rng = H.make(torch, (5,), 1, 64, "bf16", device="cpu")
    x = H.tokens(torch, rng, [1], 2, 1, 64, "bf16", device="cpu")
    c = H.cache_of(ev, t)
    ws = torch.empty(1 << 16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        ev.tree_attention(c, x["q"], x["k_new"], x["v_new"], x["tree_ptr"],
                          torch.empty_like(x["q"]), ws, 1, 5)
    with pytest.raises(ValueError):
        ev.cache_append(c, x["k_new"], x["v_new"], x["tree_ptr"], 1)
    with pytest.raises(ValueError):
        ev.cache_evict(c, 2, ws)
    # and tensors of the other place than the cache's
    d = {k: v.cuda() for k, v in t.items()}
    with pytest.raises(ValueError):
        ev.cache_append(H.cache_of(ev, d), x["k_new"], x["v_new"],
                        x["tree_ptr"].cuda(), 1)


def test_other_stream():
    import torch
    t, rng = H.make(torch, (1000,), 2, 128, "bf16", page=64, extra=40)
    x = H.tokens(torch, rng, [4], 8, 2, 128, "bf16")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        check(t, x, "bf16", decay=1.0)
    check(t, x, "bf16", decay=1.0, stream=s)


def test_captured_step_replays():
    """A step captured once (attention, append, eviction, bounds at the
    capacity) and replayed while lengths grow, against eager calls on a copy."""
    import torch
    ev = pytest.ev
    hq, hkv, d, dt = 8, 2, 128, "bf16"
    t, rng = H.make(torch, (90, 30), hkv, d, dt, page=16, extra=64)
    x = H.tokens(torch, rng, [3, 5], hq, hkv, d, dt)
    acc = torch.tensor([0, 2, 0, 1, 2, 3, 0, 0], dtype=torch.int32,
                       device="cuda")
    cnt = torch.tensor([2, 4], dtype=torch.int32, device="cuda")
    u = {k: v.clone() for k, v in t.items()}

    def step(t, out, lse, wn, ws, ws2):
        c = H.cache_of(ev, t)
        ev.tree_attention(c, x["q"], x["k_new"], x["v_new"], x["tree_ptr"],
                          out, ws, 5, c.capacity, parent=x["parent"], lse=lse,
                          decay=0.9, w_new=wn)
        ev.cache_append(c, x["k_new"], x["v_new"], x["tree_ptr"], 5,
                        accept=acc, n_accept=cnt, w_new=wn)
        ev.cache_evict(c, 100, ws2, 4, 16)

    def buffers(t):
        c = H.cache_of(ev, t)
        n = x["q"].shape[0]
        return (torch.zeros_like(x["q"]), torch.zeros(hq, n, device="cuda"),
                torch.zeros(n, hkv, device="cuda"),
                torch.zeros(ev.tree_attention_workspace(
                    c, hq, 5, c.capacity, True), dtype=torch.uint8,
                    device="cuda"),
                torch.zeros(ev.cache_evict_workspace(c, 100, c.capacity),
                            dtype=torch.uint8, device="cuda"))

    a, b = buffers(t), buffers(u)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(t, *a)
    for i in range(5):
        g.replay()
        step(u, *b)
        torch.cuda.synchronize()
        for name in t:
            assert torch.equal(t[name], u[name]), (i, name)
        for p, q in zip(a[:3], b[:3]):
            assert torch.equal(p, q), i
        x["q"].copy_(torch.randn_like(x["q"]))
        torch.cuda.synchronize()
    assert int(t["length"].max()) == 100
