"""The paged-cache operators from their definitions, in 64 bits (numpy, CPU): what
tests/test_gpu_paged*.py compare the library with."""
import numpy as np
import torch


def bf16(x):
    return torch.as_tensor(np.asarray(x)).to(torch.bfloat16)


def decode(codes, scale):
    """Values of e4m3 codes [rows, H, D] with scale bytes [H, rows], from the bits."""
    codes = np.asarray(codes).astype(np.int64)
    e, m = (codes >> 3) & 15, (codes & 7).astype(np.float64)
    mag = np.where(e == 0, m * 2.0 ** -9, np.exp2(e - 7.0) * (1 + m / 8))
    mag = np.where((codes & 127) == 127, np.nan, mag)
    val = np.where(codes >= 128, -mag, mag)
    return val * np.exp2(np.asarray(scale).astype(np.float64).T - 127)[..., None]


def scale_byte(y):
    """Scale bytes of fp32 rows y [..., D]: smallest s of 1 .. 254 with the largest
    finite magnitude at most 448 * 2^(s - 127)."""
    y = np.asarray(y, np.float64)
    mx = np.where(np.isfinite(y), np.abs(y), 0).max(-1)
    s = np.full(mx.shape, 1, np.int64)
    for v in range(2, 255):
        s = np.where(mx > 448.0 * 2.0 ** (v - 1 - 127), v, s)
    return s


def rotate(x, pos, freqs, layout, magnitude):
    """x [B, T, H, D] float64 rotated at pos [B, T]."""
    half = len(freqs)
    ang = pos[..., None].astype(np.float64) * freqs
    cs, sn = (np.cos(ang) * magnitude)[:, :, None], (np.sin(ang) * magnitude)[:, :, None]
    y = x.copy()
    ia = np.arange(half) if layout == "half" else 2 * np.arange(half)
    ib = ia + half if layout == "half" else ia + 1
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * cs - b * sn, b * cs + a * sn
    return y


def rows_of(pages, b, positions, page):
    return [int(pages[b, p // page]) * page + p % page for p in positions]


def attend(q, k, v, pages, page, lens, counts, mask, scale):
    """out, and the bounds a kernel is held to: (out, weight, score) with weight =
    sum_j p_j |v_j| + |out| per element and score = max_j scale * sum_d |q_d k_d| per
    row.  q [B, T, Hq, D], k, v [rows, Hkv, D], all float64."""
    B, T, Hq, D = q.shape
    Hkv = k.shape[1]
    out, wt = np.zeros(q.shape), np.zeros(q.shape)
    score = np.zeros(q.shape[:3])
    for b in range(B):
        n, P = int(counts[b]), int(lens[b])
        rows = rows_of(pages, b, range(P + n), page)
        for a in range(n):
            sees = np.ones(P + n, bool)
            sees[P:] = np.arange(n) <= a if mask is None else mask[b, a, :n] != 0
            r = np.asarray(rows, np.int64)[sees]
            if len(r) == 0:
                continue
            for h in range(Hq):
                kk, vv = k[r, h // (Hq // Hkv)], v[r, h // (Hq // Hkv)]
                s = kk @ q[b, a, h] * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                out[b, a, h] = p @ vv
                wt[b, a, h] = p @ np.abs(vv) + np.abs(out[b, a, h])
                score[b, a, h] = (np.abs(kk) @ np.abs(q[b, a, h])).max() * scale
    return out, wt, score


def tolerance(dtype, D, keys, out, weight, score):
    """Largest error of attend's output per element.  A score is off by at most
    (D + 8) 2^-24 of its terms' magnitudes (products, sums, scaling, the exponent's
    rounding), twice that shifts the weights; the fp32 sums add (keys + D) 2^-24 of
    the weighted magnitudes; in bf16 every weight is rounded (2^-8) and so is the
    result (2^-8)."""
    u = 2.0 ** -24
    t = weight * (2 * (D + 8) * u * score[..., None] + (keys + D) * u)
    if dtype == torch.bfloat16:
        t = t + 2.0 ** -8 * (weight + np.abs(out))
    return t + 1e-30


def backbone(B, levels, topk):
    """Parents, mask, retrieve and depth of the Backbone Expansion tree."""
    T = 1 + levels * topk
    par = np.full(T, -1)
    for i in range(1, T):
        lv = (i - 1) // topk
        par[i] = 0 if lv == 0 else 1 + (lv - 1) * topk
    mask, depth = np.zeros((T, T), np.uint8), np.zeros(T, np.int64)
    for i in range(T):
        if i:
            mask[i], depth[i] = mask[par[i]], depth[par[i]] + 1
        mask[i, i] = 1
    leaves = [i for i in range(T) if i not in par]
    ret = np.full((len(leaves), levels + 1), -1, np.int32)
    for j, i in enumerate(leaves):
        path = []
        while i >= 0:
            path.append(i)
            i = par[i]
        ret[j, :len(path)] = path[::-1]
    return par, np.tile(mask, (B, 1, 1)), np.tile(ret, (B, 1, 1)), depth


def random_tree(rng, B, T):
    mask = np.zeros((B, T, T), np.uint8)
    for b in range(B):
        for i in range(T):
            if i:
                mask[b, i] = mask[b, rng.integers(i)]
            mask[b, i, i] = 1
    return mask


def page_table(rng, need, page, spare=2):
    """Shuffled page ids for sequences of `need` positions: table, pages of the pool."""
    used = [-(-n // page) for n in need]
    ids = rng.permutation(sum(used) + spare)
    t = np.zeros((len(need), max(1, max(used))), np.int32)
    at = 0
    for b, n in enumerate(used):
        t[b, :n] = ids[at:at + n]
        at += n
    return t, sum(used) + spare
