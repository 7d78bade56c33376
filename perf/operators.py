"""The target side of a verification step, as cases that can be timed.

The drafter's tree (`Drafter.build_tree`) is verified by the target model in one
forward pass over the tree's nodes, and four operators carry a layer of that
pass: `PagedCache.append` rotates the nodes' queries and keys and writes keys
and values into the layer's paged cache (as they are, or in 8 bits),
`PagedCache.attend` lets every node attend to its sequence's prefix and to its
own ancestors, `PagedCache.gather` reads rows back as packed arrays (the form
the drafter's pass reads), and `commit_accepted` moves the accepted path's rows
behind the prefix in every layer at once.  Plain decoding (one node a sequence)
and prompt chunks (a causal run of nodes) are the same calls.

In 8 bits a row holds, per KV head, codes of float8_e4m3fn and one byte s: the
values are code * 2^(s - 127), with s the smallest of 1 .. 254 for which the
head's largest magnitude is at most 448 * 2^(s - 127).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# Query heads, KV heads, head dim of the targets the drafter shapes belong to.
HEADS = {"tiny": dict(hq=4, hkv=4, d=64), "8b": dict(hq=32, hkv=8, d=128),
         "13b": dict(hq=40, hkv=40, d=128), "70b": dict(hq=64, hkv=8, d=128)}


def _case(name, op, heads, **kw):
    c = dict(name=name, op=op, dtype="bf16", cache="bf16", batch=1, nodes=1, tree="chain", levels=0,
             topk=0, lo=0, hi=0, page=64, ragged=False)
    c.update(HEADS[heads])
    c.update(kw)
    return c


def _rope(rot, layout, theta, scaling="none"):
    return dict(rot=rot, layout=layout, theta=theta, scaling=scaling)


def _backbone(levels, topk):
    return dict(tree="backbone", levels=levels, topk=topk, nodes=1 + levels * topk)


def listed():
    return [
        # One token of each of 32 users, frequencies scaled for a long context, an
        # 8-bit cache: what every decoding step does first in every layer, all latency.
        _case("append_decode_8bit", "append", "8b", cache="f8", batch=32, lo=256, hi=8192,
              **_rope(128, "half", 500000.0, "banded")),
        # A large chunk of a long prompt (positions past 100 000), half of each head
        # rotated in neighbouring pairs.
        _case("append_prompt_8bit", "append", "70b", cache="f8", nodes=8192, lo=100000, hi=100000,
              **_rope(64, "interleaved", 500000.0, "linear")),
        # The rows of a few cycles back out of an 8-bit cache.
        _case("gather_cycle", "gather", "8b", cache="f8", batch=8, lo=1, hi=9),
        # Whole histories back out of an 8-bit cache for a batch of 32.
        _case("gather_histories", "gather", "8b", cache="f8", batch=32, lo=256, hi=8192, page=16),
        # The smallest verification: fp32, a tree of 9 nodes over 64 keys.
        _case("attend_tiny_f32", "attend", "tiny", dtype="f32", cache="f32", lo=64, hi=64, page=16,
              **_backbone(2, 4)),
        # One token of each of 32 users over ragged 8-bit histories.
        _case("attend_decode_8bit", "attend", "8b", cache="f8", batch=32, lo=256, hi=8192),
        # One user's tree on an 8B-class target: the headline cycle.
        _case("attend_tree_8b_b1", "attend", "8b", lo=1024, hi=1024, **_backbone(5, 8)),
        # A 70B-class target, 8-bit histories, a few users with trees of unequal size.
        _case("attend_tree_70b_8bit", "attend", "70b", cache="f8", batch=4, lo=1000, hi=4096, ragged=True,
              **_backbone(5, 10)),
        # The large serving batch: 32 trees of 57 nodes over ragged histories.
        _case("attend_tree_8b_b32", "attend", "8b", batch=32, lo=256, hi=8192, **_backbone(7, 8)),
        # A chunk of a long prompt behind 8192 cached positions.
        _case("attend_chunk", "attend", "8b", nodes=1024, lo=8192, hi=8192, page=256),
        # The accepted path of one user's tree, 5 layers.
        _case("commit_b1", "commit", "8b", layers=5, lo=1024, hi=1024, **_backbone(5, 8)),
        # The accepted paths of 32 users in an 8-bit cache of 32 layers.
        _case("commit_b32_8bit", "commit", "8b", cache="f8", layers=32, batch=32, lo=256, hi=1024,
              **_backbone(7, 8)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _one(rng):
    hkv = rng.choice((1, 2, 3, 4, 5, 8, 10, 40))
    group = rng.choice([g for g in (1, 2, 3, 4, 5, 7, 8) if g * hkv <= 64])
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    c = dict(op=rng.choice(("append", "gather", "attend", "attend", "attend", "commit")), dtype=dtype,
             cache="f8" if rng.random() < 0.5 else dtype, hq=hkv * group, hkv=hkv,
             d=rng.choice((64, 128, 128)), batch=_log_int(rng, 1, 64), nodes=1, tree="chain", levels=0,
             topk=0, lo=0, hi=0, page=rng.choice((16, 32, 64, 128, 1024)), ragged=rng.random() < 0.3)
    if c["op"] == "gather":
        c["hi"] = _log_int(rng, 1, 20000)
        c["lo"] = int(c["hi"] * rng.random())
        return c
    c["hi"] = _log_int(rng, 1, 32768)
    c["lo"] = int(c["hi"] * rng.random())
    if c["op"] == "commit":
        levels = rng.randint(1, 10)
        c.update(_backbone(levels, rng.randint(levels, 12)), layers=_log_int(rng, 1, 48))
        c["hi"] = min(c["hi"], 2000)
        c["lo"] = min(c["lo"], c["hi"])
        return c
    kind = rng.choice(("one", "backbone", "random", "chain"))
    if kind == "backbone":
        c.update(_backbone(rng.randint(1, 8), rng.randint(1, 10)))
    elif kind == "random":
        c.update(tree="random", nodes=_log_int(rng, 2, 130))
    elif kind == "chain":
        c["nodes"] = _log_int(rng, 2, 1024 if c["op"] == "attend" else 8192)
    if c["op"] == "append":
        c.update(_rope(16 * rng.randint(1, c["d"] // 16), rng.choice(("half", "interleaved")),
                       rng.choice((10000.0, 500000.0)),
                       rng.choice(("none", "linear", "banded", "ramp"))))
        c["batch"] = max(1, min(c["batch"], 16384 // c["nodes"]))
    return c


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        for k in w:
            most[k] = max(most.get(k, 0), w[k])
    while True:
        c = _one(rng)
        w = work(c)
        longest = c["hi"] + c["nodes"]
        padded = c["batch"] * longest  # what the plain form reads, sequences padded to the longest
        if all(w[k] <= most[k] for k in w) and padded * max(c["hkv"] * c["d"], c["hq"] * c["nodes"]) <= 6e8 \
                and c["batch"] * longest * c["hkv"] * c["d"] * c.get("layers", 1) <= 1.2e9:
            return c


def _lengths(c):
    """Prefix lengths, spread evenly over lo .. hi (prepare() shuffles them)."""
    n = c["batch"]
    if n == 1:
        return [c["hi"]]
    return [c["lo"] + round((c["hi"] - c["lo"]) * i / (n - 1)) for i in range(n)]


def _counts(c):
    """Live nodes of each sequence: all, or a few less where the batch is ragged."""
    t = c["nodes"]
    return [max(1, t - (3 * i) % max(1, (t + 1) // 2)) if c["ragged"] else t for i in range(c["batch"])]


def _row_bytes(c, kind):
    per = {"f32": 4, "bf16": 2, "f8": 1}[kind]
    return 2 * c["hkv"] * (c["d"] * per + (1 if kind == "f8" else 0))


def work(c):
    es = {"f32": 4, "bf16": 2}[c["dtype"]]
    lens, counts = _lengths(c), _counts(c)
    live = sum(counts)
    qd = c["hq"] * c["d"]
    if c["op"] == "append":
        b = live * (2 * qd * es + _row_bytes(c, c["dtype"]) + _row_bytes(c, c["cache"]))
        if c["cache"] == "f8":
            b += live * (_row_bytes(c, "f8") + _row_bytes(c, c["dtype"]))
        return {"bytes": b, "flops": 3 * live * (c["hq"] + c["hkv"]) * c["rot"]}
    if c["op"] == "gather":
        n = max(1, sum(lens))
        return {"bytes": n * (_row_bytes(c, c["cache"]) + _row_bytes(c, c["dtype"])), "flops": n * c["hkv"] * c["d"]}
    if c["op"] == "commit":
        moved = sum(_accepted(c))
        return {"bytes": 2 * max(1, moved) * _row_bytes(c, c["cache"]) * c["layers"], "flops": 0}
    pairs = 0
    for p, n in zip(lens, counts):
        inner = n * (n + 1) // 2
        if c["tree"] == "backbone":  # a node sees itself, the root and the backbone before it
            inner = 1 + sum(2 + (i - 1) // c["topk"] for i in range(1, n))
        elif c["tree"] == "random":  # ancestors of a node in a random tree: about log of its index
            inner = sum(1 + int(math.log(i + 1)) for i in range(n))
        pairs += p * n + inner
    b = (sum(lens) + live) * _row_bytes(c, c["cache"]) + 2 * live * qd * es
    return {"bytes": b + (c["batch"] * c["nodes"] ** 2 if c["tree"] != "chain" else 0),
            "flops": 4 * pairs * qd}


def _accepted(c):
    """Accepted nodes of each sequence, 0 .. levels in turn, deep ones more often."""
    return [c["levels"] - (i * 7) % (c["levels"] + 1) for i in range(c["batch"])]


def frequencies(c):
    """Radians per position of every rotated pair, and the factor on cosine and
    sine: the published scalings for contexts longer than the trained one."""
    half, theta = c["rot"] // 2, c["theta"]
    w = [theta ** (-2.0 * m / c["rot"]) for m in range(half)]
    if c["scaling"] == "linear":
        return [x / 8.0 for x in w], 1.0
    if c["scaling"] == "banded":  # by wavelength: long ones slowed down by 8, short ones kept
        out = []
        for x in w:
            turns = 8192.0 * x / (2 * math.pi)  # over the trained context
            s = min(1.0, max(0.0, (turns - 1.0) / (4.0 - 1.0)))
            out.append((1 - s) * x / 8.0 + s * x)
        return out, 1.0
    if c["scaling"] == "ramp":  # by the pair's index, with a factor on the result

        def pair(turns):
            return c["rot"] * math.log(4096.0 / (turns * 2 * math.pi)) / (2 * math.log(theta))
        low, high = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), half - 1)
        high = high if high > low else low + 0.001
        s = [min(1.0, max(0.0, (m - low) / (high - low))) for m in range(half)]
        return [x / 16.0 * r + x * (1 - r) for x, r in zip(w, s)], 0.1 * math.log(16.0) + 1.0
    return w, 1.0


def _trees(c, rnd):
    """Parents of every sequence's nodes, [B, T] (-1: the root)."""
    par = np.full((c["batch"], c["nodes"]), -1, np.int64)
    for b in range(c["batch"]):
        for i in range(1, c["nodes"]):
            if c["tree"] == "backbone":
                level = (i - 1) // c["topk"]
                par[b, i] = 0 if level == 0 else 1 + (level - 1) * c["topk"]
            else:
                par[b, i] = rnd.randrange(i)
    return par


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rnd = random.Random(int(seed))
    t, b, hkv, d, page = c["nodes"], c["batch"], c["hkv"], c["d"], c["page"]
    dt = TYPES[c["dtype"]]
    lens = _lengths(c)
    rnd.shuffle(lens)
    per_seq = -(-(c["hi"] + t) // page)
    used = [-(-(p + t) // page) for p in lens]
    n_pages = sum(used) + 3
    ids = list(range(n_pages))
    rnd.shuffle(ids)
    table = np.zeros((b, per_seq), np.int32)
    at = 0
    for i, n in enumerate(used):
        table[i, :n] = ids[at:at + n]
        at += n

    def dev(a, kind=torch.int32):
        return torch.tensor(np.asarray(a), dtype=kind, device=DEV)

    def normal(*shape, scale=1.0, kind=dt):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * scale).to(kind)

    st = dict(c=c, pages=dev(table), lens=dev(lens), page=page)
    layers = c.get("layers", 1)
    rows = n_pages * page
    kind = {"f8": torch.uint8, "bf16": torch.bfloat16, "f32": torch.float32}[c["cache"]]
    pools = []
    for _ in range(layers):
        pool = {}
        for n in ("k", "v"):
            if c["op"] == "append":
                pool[n] = torch.zeros((rows, hkv, d), dtype=kind, device=DEV)
            else:
                pool[n] = normal(rows, hkv, d, kind=torch.float32)
                if c["cache"] == "f8":  # as the cache holds them: magnitudes up to 448
                    pool[n] = (pool[n] * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                else:
                    pool[n] = pool[n].to(kind)
            if c["cache"] == "f8":  # 100 * 2^-7 and its neighbours: values around 1
                s = torch.randint(119, 122, (hkv, rows), generator=g, device=DEV, dtype=torch.int32)
                pool[n + "_scale"] = (s * (c["op"] != "append")).to(torch.uint8)
        pools.append(pool)
    st["pools"] = pools
    counts = _counts(c)
    st["counts"] = dev(counts) if c["ragged"] and c["op"] in ("append", "attend") else None
    if c["op"] == "gather":
        # from position 0 of every sequence; the packed rows of the drafter's prefix caches
        st["n_rows"] = sum(lens)
        st["cu"] = dev(np.concatenate([[0], np.cumsum(lens)]))
        st["out"] = [torch.zeros((st["n_rows"], hkv, d), dtype=dt, device=DEV) for _ in range(2)]
    elif c["op"] == "append":
        # queries, keys and values side by side, as one projection leaves them
        qkv = normal(b, t, (c["hq"] + 2 * hkv) * d)
        qe, ke = c["hq"] * d, (c["hq"] + hkv) * d
        st["q"], st["k"], st["v"] = (x.unflatten(2, (-1, d)) for x in
                                     (qkv[..., :qe], qkv[..., qe:ke], qkv[..., ke:]))
        depth = np.tile(np.arange(t), (b, 1))
        if c["tree"] != "chain":
            par = _trees(c, rnd)
            for i in range(t):
                depth[:, i] = np.where(par[:, i] < 0, 0, depth[np.arange(b), par[:, i]] + 1)
        st["positions"] = dev(np.asarray(lens)[:, None] + depth)
        w, mag = frequencies(c)
        st["freqs"], st["magnitude"] = dev(w, torch.float64), mag
        st["q_out"] = torch.zeros((b, t, c["hq"], d), dtype=dt, device=DEV)
        if c["cache"] == "f8":
            st["cu"] = dev(np.concatenate([[0], np.cumsum(counts)]))
            st["n_rows"] = sum(counts)
            st["back"] = [torch.zeros((st["n_rows"], hkv, d), dtype=dt, device=DEV) for _ in range(2)]
    elif c["op"] == "attend":
        st["q"] = normal(b, t, c["hq"], d, scale=2.5)  # scores of a few units: neither flat nor one key
        st["out"] = torch.zeros((b, t, c["hq"], d), dtype=dt, device=DEV)
        st["mask"] = None
        if c["tree"] != "chain":
            par = _trees(c, rnd)
            m = np.zeros((b, t, t), np.uint8)
            for i in range(t):
                m[:, i] = np.where(par[:, i, None] < 0, 0, m[np.arange(b), par[:, i]])
                m[:, i, i] = 1
            st["mask"] = dev(m, torch.uint8)
    else:
        n, k = c["levels"], c["topk"]
        paths = [[0] + [1 + lv * k for lv in range(n)]]  # the backbone, then its side branches
        for lv in range(n):
            for r in range(1, k):
                p = [0] + [1 + x * k for x in range(lv)] + [1 + lv * k + r]
                paths.append(p + [-1] * (n + 1 - len(p)))
        acc = _accepted(c)
        rnd.shuffle(acc)
        # the accepted nodes: the backbone, or a side branch at the last of them
        path = [0 if a == 0 or rnd.random() < 0.5 else 1 + (a - 1) * (k - 1) + rnd.randrange(k - 1)
                if k > 1 else 0 for a in acc]
        st["retrieve"] = dev(np.tile(np.asarray(paths), (b, 1, 1)))
        st["accept_len"], st["accept_path"] = dev(acc), dev(path)
        st["new_lens"] = torch.zeros(b, dtype=torch.int32, device=DEV)
    st["handle"] = None
    return st


def _caches(st):
    """The program's handles on its caches, made once and kept with them."""
    if st["handle"] is None:
        from paper_2509_20416_amd import PagedCache
        st["handle"] = [PagedCache(p["k"], p["v"], st["page"], p.get("k_scale"), p.get("v_scale"))
                        for p in st["pools"]]
    return st["handle"]


def _run_own(st):
    c, caches = st["c"], _caches(st)
    cache = caches[0]
    if c["op"] == "append":
        from paper_2509_20416_amd import Rope
        rope = Rope(st["freqs"], layout=c["layout"], magnitude=st["magnitude"])
        cache.append(st["pages"], st["lens"], st["k"], st["v"], positions=st["positions"], counts=st["counts"],
                     rope=rope, q=st["q"], q_out=st["q_out"])
        if c["cache"] != "f8":
            return {"q": st["q_out"], "k": st["pools"][0]["k"], "v": st["pools"][0]["v"]}
        k, v = cache.gather(st["pages"], st["cu"], st["n_rows"], starts=st["lens"], out=st["back"])
        return {"q": st["q_out"], "k": k, "v": v}
    if c["op"] == "gather":
        k, v = cache.gather(st["pages"], st["cu"], st["n_rows"], out=st["out"])
        return {"k": k, "v": v}
    if c["op"] == "attend":
        if "workspace" not in st:
            st["workspace"] = cache.attend_workspace(c["batch"], c["nodes"], c["hq"], c["hi"] + c["nodes"],
                                                     dtype=st["q"].dtype)
        return {"out": cache.attend(st["pages"], st["lens"], st["q"], mask=st["mask"], counts=st["counts"],
                                    max_len=c["hi"] + c["nodes"], out=st["out"], workspace=st["workspace"])}
    from paper_2509_20416_amd import commit_accepted
    commit_accepted(caches, st["pages"], st["lens"], st["retrieve"], st["accept_path"], st["accept_len"],
                    nodes=c["nodes"], new_lens=st["new_lens"])
    return _committed(st)


def _committed(st):
    """The lengths, and the cache of the first and the last layer."""
    return {"lens": st["new_lens"], "first": _values(st["pools"][0], st["c"]),
            "last": _values(st["pools"][-1], st["c"])}


def _values(pool, c):
    """What a commit leaves: values as they are held (8-bit codes as the floats
    they are, beside their scale bytes)."""
    if c["cache"] != "f8":
        return [pool["k"], pool["v"]]
    return [pool["k"].view(torch.float8_e4m3fn), pool["v"].view(torch.float8_e4m3fn), pool["k_scale"],
            pool["v_scale"]]


# ---- plain forms ---------------------------------------------------------------


def _rows_of(st, pos):
    """Cache rows of positions pos [B, n] of every sequence."""
    page = st["page"]
    idx = torch.clamp(torch.div(pos, page, rounding_mode="floor"), 0, st["pages"].shape[1] - 1)
    return torch.gather(st["pages"].long(), 1, idx) * page + pos % page


def _read(pool, name, rows):
    """fp32 values of cache rows, whatever they are held in."""
    x = pool[name][rows]
    if name + "_scale" not in pool:
        return x.float()
    s = pool[name + "_scale"].t()[rows].int()
    return x.view(torch.float8_e4m3fn).float() * (s << 23).view(torch.float32)[..., None]


def _quantise(y):
    """Codes (as bytes) and scale bytes of fp32 values y [..., D]."""
    mag = torch.where(torch.isfinite(y), y.abs(), 0.0).amax(-1)
    f, e = torch.frexp(mag)
    s = torch.where(mag > 0, e - 9 + 127 + (f > 0.875).int(), 1).clamp(1, 254)
    codes = (y * ((254 - s) << 23).view(torch.float32)[..., None]).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), s.to(torch.uint8)


def _rotate(x, ang, mag, rot, layout):
    """x [B, T, H, D] rotated by ang [B, T, rot / 2], in 64 bits."""
    x = x.double()
    cos, sin = (torch.cos(ang) * mag)[:, :, None], (torch.sin(ang) * mag)[:, :, None]
    head = x[..., :rot]
    if layout == "half":
        a, b = head[..., :rot // 2], head[..., rot // 2:]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(st):
    c, pool, dt = st["c"], st["pools"][0], TYPES[st["c"]["dtype"]]
    t = c["nodes"]
    node = torch.arange(t, device=DEV)
    live = node[None] < (st["counts"][:, None] if st["counts"] is not None else torch.full_like(st["lens"], t)[:, None])
    ang = st["positions"].double()[..., None] * st["freqs"]
    q = _rotate(st["q"], ang, st["magnitude"], c["rot"], c["layout"]).float().to(dt)
    q = torch.where(live[..., None, None], q, st["q_out"])
    k = _rotate(st["k"], ang, st["magnitude"], c["rot"], c["layout"]).float()
    rows = _rows_of(st, st["lens"].long()[:, None] + node[None])[live]
    back = []
    for n, x in (("k", k), ("v", st["v"].float())):
        x = x[live]
        if c["cache"] == "f8":
            codes, s = _quantise(x)
            pool[n][rows] = codes
            pool[n + "_scale"][:, rows] = s.t()
            back.append(_read(pool, n, rows).to(dt))
        else:
            pool[n][rows] = x.to(pool[n].dtype)
            back.append(pool[n])
    return {"q": q, "k": back[0], "v": back[1]}


def _plain_gather(st):
    c, dt = st["c"], TYPES[st["c"]["dtype"]]
    r = torch.arange(st["n_rows"], device=DEV)
    seq = torch.searchsorted(st["cu"][1:].long(), r, right=True)
    pos = r - st["cu"].long()[seq]
    rows = st["pages"].long()[seq, torch.div(pos, st["page"], rounding_mode="floor")] * st["page"] + pos % st["page"]
    return {n: _read(st["pools"][0], n, rows).to(dt) for n in ("k", "v")}


def _plain_attend(st):
    c, t, d = st["c"], st["c"]["nodes"], st["c"]["d"]
    b, hkv, grp = c["batch"], c["hkv"], c["hq"] // c["hkv"]
    longest = c["hi"] + t
    key = torch.arange(longest, device=DEV)[None].expand(b, -1)
    lens = st["lens"].long()[:, None]
    counts = st["counts"].long()[:, None] if st["counts"] is not None else torch.full_like(lens, t)
    inside = key < lens + counts
    rows = _rows_of(st, key)
    k = _read(st["pools"][0], "k", rows).permute(0, 2, 3, 1).contiguous()    # [B, Hkv, D, L]
    q = st["q"].float().reshape(b, t, hkv, grp, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, t * grp, d)
    s = torch.matmul(q, k) * (1.0 / math.sqrt(d))
    del k
    node = key - lens
    if st["mask"] is None:
        own_part = node[:, None] <= torch.arange(t, device=DEV)[None, :, None]
    else:
        own_part = torch.gather(st["mask"], 2, node.clamp(0, t - 1)[:, None].expand(-1, t, -1)) != 0
    sees = ((node < 0)[:, None] | own_part) & inside[:, None]                 # [B, T, L]
    s = s.view(b, hkv, t, grp, longest).masked_fill_(~sees[:, None, :, None], float("-inf"))
    p = torch.exp_(s - s.amax(-1, keepdim=True))
    p = p.div_(p.sum(-1, keepdim=True)).view(b, hkv, t * grp, longest)
    v = _read(st["pools"][0], "v", rows)
    v = torch.where(inside[..., None, None], v, 0.0).permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p, v).view(b, hkv, t, grp, d).permute(0, 2, 1, 3, 4).reshape(b, t, c["hq"], d)
    live = torch.arange(t, device=DEV)[None] < counts
    return {"out": torch.where(live[..., None, None], o.to(st["out"].dtype), st["out"])}


def _plain_commit(st):
    c = st["c"]
    b, n = c["batch"], c["levels"]
    path = st["retrieve"][torch.arange(b, device=DEV), st["accept_path"].long()].long()  # [B, N+1]
    depth = torch.arange(n + 1, device=DEV)[None]
    moved = (depth >= 1) & (depth <= st["accept_len"][:, None])
    lens = st["lens"].long()[:, None]
    src = _rows_of(st, lens + torch.where(moved, path, 0))[moved]
    dst = _rows_of(st, lens + depth.expand(b, -1))[moved]
    [_move(p, src, dst) for p in st["pools"]]
    st["new_lens"].copy_(st["lens"] + 1 + st["accept_len"])
    return _committed(st)


def _move(pool, src, dst):
    for n in ("k", "v"):
        pool[n][dst] = pool[n][src]
        if n + "_scale" in pool:
            pool[n + "_scale"][:, dst] = pool[n + "_scale"][:, src]


def run(st):
    if own:
        return _run_own(st)
    op = st["c"]["op"]
    return {"append": _plain_append, "gather": _plain_gather, "attend": _plain_attend,
            "commit": _plain_commit}[op](st)


# ---- from the definitions, in 64 bits, a sequence at a time ---------------------


def _held(pool, name, row):
    """64-bit values of cache rows: 1 sign, 4 exponent (bias 7), 3 mantissa bits
    and the scale byte's power of two, or the stored numbers."""
    x = pool[name][row]
    if name + "_scale" not in pool:
        return x.double()
    x = x.long()
    e, m = (x >> 3) & 15, (x & 7).double()
    mag = torch.where(e == 0, m / 512.0, torch.exp2(e.double() - 7.0) * (1.0 + m / 8.0))
    mag = torch.where((x & 127) == 127, torch.full_like(mag, math.nan), mag)
    power = torch.exp2(pool[name + "_scale"][:, row].double().t() - 127.0)
    return torch.where(x >= 128, -mag, mag) * power[..., None]


def _rows_1(st, i, p0, p1):
    pos = torch.arange(p0, p1, device=DEV)
    return st["pages"][i].long()[pos // st["page"]] * st["page"] + pos % st["page"]


def _nearest_8bit(y):
    """What an 8-bit head holds for the 64-bit values y [n, H, D] (rounded to 32
    bits first, as the definition has it)."""
    y = y.float().double()
    top = y.abs().amax(-1, keepdim=True)
    s = torch.full_like(top, -126.0)
    big = top > 448.0 * 2.0 ** -126
    guess = torch.ceil(torch.log2(torch.where(big, top, 1.0) / 448.0))
    guess = torch.where(top > 448.0 * torch.exp2(guess), guess + 1, guess)
    guess = torch.where(top <= 448.0 * torch.exp2(guess - 1), guess - 1, guess)
    s = torch.where(big, guess.clamp(min=-126), s)
    z = y / torch.exp2(s)
    e = torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -9))).clamp(min=-6)
    e = torch.where(z.abs() >= torch.exp2(e + 1), e + 1, e)
    step = torch.exp2(e - 3)
    return torch.round(z / step) * step * torch.exp2(s)  # torch.round: ties to even


def _exact_append(st):
    c = st["c"]
    half, mag, h = c["rot"] // 2, st["magnitude"], c["rot"]
    counts = _counts(c)
    # complex numbers: a pair (a, b) times magnitude * exp(i angle)
    turn = torch.polar(torch.full((), mag, dtype=torch.float64, device=DEV),
                       st["positions"].double()[..., None] * st["freqs"])[:, :, None]

    def rotated(x):
        y = x.double().clone()
        at = (slice(0, half), slice(half, h)) if c["layout"] == "half" else (slice(0, h, 2), slice(1, h, 2))
        z = torch.complex(y[..., at[0]], y[..., at[1]]) * turn
        y[..., at[0]], y[..., at[1]] = z.real, z.imag
        return y
    q = st["q_out"].double().clone()
    rq, rk = rotated(st["q"]), rotated(st["k"])
    pools = {n: st["pools"][0][n].double() for n in ("k", "v")} if c["cache"] != "f8" else None
    back = {"k": [], "v": []}
    for i, n in enumerate(counts):
        q[i, :n] = rq[i, :n]
        p = int(st["lens"][i])
        for name, x in (("k", rk[i, :n]), ("v", st["v"][i, :n].double())):
            if pools is None:
                back[name].append(_nearest_8bit(x))
            else:
                pools[name][_rows_1(st, i, p, p + n)] = x
    got = pools if pools is not None else {n: torch.cat(x) for n, x in back.items()}
    return {"q": q, "k": got["k"], "v": got["v"]}


def _exact_attend(st):
    c, t, d = st["c"], st["c"]["nodes"], st["c"]["d"]
    grp = c["hq"] // c["hkv"]
    out = st["out"].double().clone()
    lens, counts = st["lens"].tolist(), _counts_now(st)
    for i in range(c["batch"]):
        n, p = counts[i], lens[i]
        rows = _rows_1(st, i, 0, p + n)
        k, v = (_held(st["pools"][0], x, rows) for x in ("k", "v"))
        sees = torch.ones(n, p + n, dtype=torch.bool, device=DEV)
        if st["mask"] is None:
            sees[:, p:] = torch.tril(sees[:, p:])
        else:
            sees[:, p:] = st["mask"][i, :n, :n] != 0
        for h in range(c["hkv"]):
            q = st["q"][i, :n, h * grp:(h + 1) * grp].double().reshape(n * grp, d)
            s = (q @ k[:, h].t().contiguous()) / math.sqrt(d)
            s = s.view(n, grp, -1).masked_fill(~sees[:, None], -math.inf)
            out[i, :n, h * grp:(h + 1) * grp] = (torch.softmax(s, -1).view(n * grp, -1) @ v[:, h].contiguous()).view(n, grp, d)
    return {"out": out}


def _counts_now(st):
    return st["counts"].tolist() if st["counts"] is not None else [st["c"]["nodes"]] * st["c"]["batch"]


def exact(c, seed):
    if c["op"] == "attend" and work(c)["flops"] > 1e12:
        return None
    st = prepare(c, seed)
    if c["op"] == "append":
        return _exact_append(st)
    if c["op"] == "attend":
        return _exact_attend(st)
    if c["op"] == "gather":
        rows = torch.cat([_rows_1(st, i, 0, int(n)) for i, n in enumerate(st["lens"])])
        return {n: _held(st["pools"][0], n, rows) for n in ("k", "v")}
    lens, acc = st["lens"].tolist(), st["accept_len"].tolist()
    for i in range(c["batch"]):
        path = st["retrieve"][i, int(st["accept_path"][i])].tolist()
        for pool in (st["pools"][0], st["pools"][-1]):
            if pool is st["pools"][-1] and pool is st["pools"][0] and pool.get("done") == i:
                continue
            pool["done"] = i
            for step in range(1, acc[i] + 1):
                a, z = (int(_rows_1(st, i, lens[i] + x, lens[i] + x + 1)) for x in (path[step], step))
                for n in ("k", "v"):
                    pool[n][z] = pool[n][a]
                    if n + "_scale" in pool:
                        pool[n + "_scale"][:, z] = pool[n + "_scale"][:, a]
    st["new_lens"].copy_(torch.tensor([p + 1 + a for p, a in zip(lens, acc)]))
    got = _committed(st)
    return {"lens": None, **{n: [x.double() if x.is_floating_point() else None for x in got[n]] for n in ("first", "last")}}
