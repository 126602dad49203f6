"""Random caches and trees for the cache tests: torch tensors for the library
and their fp64 images for the oracle."""
from __future__ import annotations

import numpy as np


def make(torch, lens, hkv, d, dtype, page=16, layout="token", extra=0,
         device="cuda", seed=0, evicted=0):
    """(cache tensors, generator). ``extra``: tokens that every sequence has
    room for beyond its length; ``evicted``: positions gone from the front."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    used = [-(-(x + extra) // page) for x in lens]
    max_pages = max(1, max(used))
    n_pages = sum(used) + 2
    table = np.full((n, max_pages), -1, np.int32)
    order = rng.permutation(n_pages)
    at = 0
    for i, u in enumerate(used):
        table[i, :u] = order[at:at + u]
        at += u
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def pool():
        x = rng.standard_normal((n_pages, page, hkv, d)).astype(np.float32)
        x = torch.from_numpy(x).to(dt)
        if layout == "head":
            x = x.transpose(1, 2).contiguous().transpose(1, 2)
        elif layout == "wide":    # rows inside wider ones (K and V side by side)
            w = torch.full((n_pages, page, hkv, d + 16), 7.0, dtype=dt)
            w[..., :d] = x
            x = w
        x = x.to(device)
        return x[..., :d]

    cap = max_pages * page
    t = {"k": pool(), "v": pool(),
         "page_table": torch.from_numpy(table).to(device),
         "length": torch.tensor(lens, dtype=torch.int32, device=device),
         "seen": torch.tensor([x + evicted for x in lens], dtype=torch.int32,
                              device=device)}
    w = np.exp(1.5 * rng.standard_normal((n, hkv, cap))).astype(np.float32)
    w[rng.random(w.shape) < 0.2] = 0
    t["weight"] = torch.from_numpy(w).to(device)
    pos = np.stack([np.stack([np.concatenate(
        [rng.permutation(x + evicted)[:x],
         np.full(cap - x, -5)]) for _ in range(hkv)]) for x in lens])
    t["pos"] = torch.from_numpy(pos.astype(np.int32)).to(device)
    return t, rng


def host(t):
    """Arrays of a cache's tensors (fp64 for floating ones)."""
    return {k: (x.detach().cpu().double().numpy()
                if x.is_floating_point() else x.cpu().numpy())
            for k, x in t.items() if x is not None}


def tokens(torch, rng, ns, hq, hkv, d, dtype, slack=0, device="cuda",
           scale=1.0):
    """q, k_new, v_new, tree_ptr and random parents of trees of ns tokens;
    ``slack``: rows behind the last sequence's."""
    total = sum(ns) + slack
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rows(h, s=1.0):
        x = (s * rng.standard_normal((total, h, d))).astype(np.float32)
        return torch.from_numpy(x).to(dt).to(device)

    ptr = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
    parent = np.full(total, -1, np.int32)
    for a, n in zip(ptr, ns):
        for i in range(1, n):
            parent[a + i] = rng.integers(max(-1, i - 6), i)
    return {"q": rows(hq, scale), "k_new": rows(hkv), "v_new": rows(hkv),
            "tree_ptr": torch.from_numpy(ptr).to(device),
            "parent": torch.from_numpy(parent).to(device)}


def cache_of(ev, t):
    return ev.Cache(t["k"], t["v"], t["page_table"], t["length"],
                    seen=t.get("seen"), weight=t.get("weight"),
                    pos=t.get("pos"))


def tolerances(ref, d, dtype, keys, rows, decay=1.0, weight0=None):
    """Bounds of each output's distance from the oracle's.

    u = 2^-24 is half a step of fp32. A logit is a sum of d products of exact
    inputs in fp32, scaled once (and once more into log2 units), so it is off
    by at most (d + 4) u times the sum of |q||k| * scale; in the exponential
    that is a relative error, ds, doubled as the row's sum has it too (exp2
    itself: 4u). Sums of N terms add N u. bf16: each probability and the
    output are rounded by half a step, 2^-8 of the value."""
    u = 2.0 ** -24
    ds = 2 * (d + 4) * u * ref["absqk"] + 8 * u
    rel = ds + 2 * (keys + 16) * u
    half = 2.0 ** -8 if dtype == "bf16" else u
    out = (rel[..., None] + (half if dtype == "bf16" else 0)) * ref["absv"] \
        + half * np.abs(np.nan_to_num(ref["out"]))
    lse = (ds + (keys + 16) * u).T + 4 * u * np.abs(
        np.nan_to_num(ref["lse"], neginf=0.0))
    mrel = 2 * ds.max(initial=0.0) + (2 * keys + rows + 32) * u
    weight = 2 * u * np.abs(ref["weight"]) + mrel * ref["mass"] + 1e-30
    if weight0 is not None:
        weight = weight + 2 * u * np.abs(decay * weight0)
    w_new = (mrel + 2 * u) * np.abs(np.nan_to_num(ref["w_new"])) + 1e-30
    return {"out": out + 1e-30, "lse": lse, "weight": weight, "w_new": w_new}


def close(name, got, want, tol, where=None):
    """got within tol of want, NaN and infinities in the same places."""
    g, w = np.asarray(got, np.float64), np.asarray(want, np.float64)
    if where is not None:
        g, w, tol = g[where], w[where], tol[where]
    fin = np.isfinite(w)
    assert np.array_equal(np.isnan(g), np.isnan(w)), f"{name}: NaN elsewhere"
    assert np.array_equal(g[~fin & ~np.isnan(w)], w[~fin & ~np.isnan(w)]), \
        f"{name}: infinities elsewhere"
    err = np.abs(g[fin] - w[fin])
    bad = err > tol[fin]
    assert not bad.any(), (
        f"{name}: {int(bad.sum())} of {bad.size} off by up to "
        f"{float((err / tol[fin]).max()):.2f} times the tolerance")
