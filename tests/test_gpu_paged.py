"""GPU parity of the paged-cache operators (append, gather, attend, commit) with
plain 64-bit implementations (tests/paged_ref.py)."""
import numpy as np
import pytest
import torch

from tests import paged_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def dev(a, dt=torch.int32):
    return torch.as_tensor(np.asarray(a)).to(dt).to(DEV)


def f64(t):
    return t.detach().double().cpu().numpy()


def make_cache(rng, n_pages, page, hkv, D, kind, fill=True):
    """A PagedCache of normal values (garbage scales where not filled)."""
    from paper_2509_20416_amd import PagedCache
    c = PagedCache.empty(n_pages, page, hkv, D, kind, DEV)
    rows = n_pages * page
    for t, s in ((c.k, c.k_scale), (c.v, c.v_scale)):
        x = torch.as_tensor(rng.standard_normal((rows, hkv, D)), dtype=F32)
        if kind == F8:
            t.view(torch.uint8).copy_((x * 100).clamp(-448, 448).to(F8).view(torch.uint8))
            s.copy_(dev(rng.integers(119, 122, (hkv, rows)), torch.uint8))
        else:
            t.copy_(x.to(kind))
    return c


def held(c, which):
    """float64 values of every row of the cache's keys or values."""
    t, s = (c.k, c.k_scale) if which == "k" else (c.v, c.v_scale)
    if s is None:
        return f64(t)
    return R.decode(t.view(torch.uint8).cpu().numpy(), s.cpu().numpy())


# ---- append ---------------------------------------------------------------------


@pytest.mark.parametrize("dt,kind", [(BF, BF), (BF, F8), (F32, F32), (F32, F8)])
@pytest.mark.parametrize("D,rot,layout", [(128, 128, "half"), (128, 48, "half"), (64, 16, "interleaved"),
                                          (64, 64, "interleaved"), (128, 112, "interleaved"), (64, 32, "half")])
def test_append(dt, kind, D, rot, layout):
    from paper_2509_20416_amd import Rope, fe
    rng = np.random.default_rng(D + rot + (dt == BF))
    B, T, Hq, Hkv, page = 3, 5, 6, 3, 16
    starts, counts = np.array([0, 29, 1000]), np.array([5, 3, 4])
    pages, n_pages = R.page_table(rng, [1005] * 3, page)
    c = make_cache(rng, n_pages, page, Hkv, D, kind)
    before = {n: held(c, n) for n in "kv"}
    freqs, mag = fe.fe_rope_frequencies(rot, 10000.0, fe.FE_SCALE_RAMP, 4.0, 1.0, 32.0, 4096.0)
    x = torch.as_tensor(rng.standard_normal((B, T, Hq + 2 * Hkv, D)) * 3, dtype=F32).to(dt).to(DEV)
    q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]   # rows of a joint projection
    pos = np.array([[0, 1, 1, 2, 3], [30, 31, 32, 33, 34], [131000, 131001, 131001, 500000, 9]])
    q_out = torch.full((B, T, Hq, D), 7.0, dtype=dt, device=DEV)
    got = c.append(dev(pages), dev(starts), k, v, positions=dev(pos), counts=dev(counts),
                   rope=Rope(dev(freqs, torch.float64), layout, mag), q=q, q_out=q_out)
    assert got is q_out
    u = 2.0 ** -24
    want_q, want_k, want_v = R.rotate(f64(q), pos, freqs, layout, mag), R.rotate(f64(k), pos, freqs, layout, mag), f64(v)
    size = np.abs(f64(x)).max() * mag
    # one rounding to the result's type; in bf16 the rotation is fp32: rounded sine, cosine, product, sum
    step = {BF: 2.0 ** -8, F32: u}[dt]
    arith = 6 * u * size if dt == BF else 1e-12
    gq = f64(q_out)
    for b in range(B):
        n = counts[b]
        assert np.all(np.abs(gq[b, :n] - want_q[b, :n]) <= step * np.abs(want_q[b, :n]) * (1 + 1e-6) + arith)
        assert np.all(gq[b, n:] == 7.0)
    touched = {n: np.zeros(before[n].shape[0], bool) for n in "kv"}
    after = {n: held(c, n) for n in "kv"}
    for name, want in (("k", want_k), ("v", want_v)):
        for b in range(B):
            n = counts[b]
            rows = R.rows_of(pages, b, range(starts[b], starts[b] + n), page)
            touched[name][rows] = True
            w, g = want[b, :n], after[name][rows]
            if kind == F8:
                s = R.scale_byte(w.astype(np.float32))
                sc = (c.k_scale if name == "k" else c.v_scale).cpu().numpy()[:, rows].T
                assert np.array_equal(s, sc)
                # half a step: 2^-4 of the value, 2^-10 of the scale among the smallest codes
                assert np.all(np.abs(g - w) <= np.maximum(2.0 ** -4 * np.abs(w), 2.0 ** -10 * np.exp2(s - 127.0)[..., None]) * (1 + 1e-6))
            else:
                assert np.all(np.abs(g - w) <= step * np.abs(w) * (1 + 1e-6) + (arith if name == "k" else 0))
        assert np.array_equal(after[name][~touched[name]], before[name][~touched[name]])


def test_append_codes_exactly():
    """Values (unrotated) against torch's own e4m3 rounding, bit for bit: scale
    borders, ties, zero rows, subnormal codes, the largest floats, infinities, NaN."""
    rng = np.random.default_rng(5)
    D, page = 64, 16
    x = rng.standard_normal((16, D)).astype(np.float32)
    x[1] = 0
    x[2, 0] = 448.0 * 4
    x[2, 1:] = 0.013
    x[3, 0] = np.nextafter(np.float32(448.0 * 4), np.float32(1e9))
    x[4] = np.arange(D) * 2.0 ** -9 / 2          # halves of the smallest step, ties among them
    x[4, 63] = 448
    x[5, 3], x[5, 4], x[5, 5] = np.inf, -np.inf, np.nan
    x[6] = np.nan
    x[7] = 3e38 * np.linspace(-1, 1, D)
    x[8] = 2.0 ** -126 * np.linspace(0, 1, D)
    x[9] = 1e-42
    x[10, :] = 17.0 + np.arange(D) % 4 * 0.5      # ties between codes
    x[10, 0] = 448
    c = make_cache(rng, 2, page, 1, D, F8)
    t = torch.as_tensor(x).to(DEV).view(1, 16, 1, D)
    c.append(dev([[1, 0]]), dev([0]), t, t)
    s = R.scale_byte(x)
    y = np.where(np.isfinite(x), x, np.nan).astype(np.float64) * np.exp2(127.0 - s)[:, None]
    want = torch.as_tensor(y.astype(np.float32)).to(F8).view(torch.uint8).numpy()
    for codes, sc in ((c.k, c.k_scale), (c.v, c.v_scale)):
        g = codes.view(torch.uint8).cpu().numpy()[16:, 0]
        assert np.array_equal(sc.cpu().numpy()[0, 16:], s)
        nan = np.isnan(y)
        assert np.array_equal(g[~nan], want[~nan])
        assert np.all((g[nan] & 127) == 127)


def test_append_leaves_bad_rows():
    """Positions and pages out of range: nothing written, the queries still turned."""
    from paper_2509_20416_amd import Rope, fe
    rng = np.random.default_rng(6)
    c = make_cache(rng, 4, 16, 2, 64, BF)
    before = c.k.clone(), c.v.clone()
    pages = np.array([[0, 1], [-1, 4], [2, 3]])
    x = torch.randn(3, 3, 2, 64, device=DEV, dtype=BF)
    freqs, _ = fe.fe_rope_frequencies(64, 10000.0)
    out = c.append(dev(pages), dev([-1, 15, 30]), x, x, rope=Rope(dev(freqs, torch.float64)), q=x)
    pos = np.array([-1, 15, 30])[:, None] + np.arange(3)
    want = R.rotate(f64(x), pos, freqs, "half", 1.0)
    assert np.all(np.abs(f64(out) - want) <= 2.0 ** -8 * np.abs(want) + 1e-5)
    new = {2 * 16 + 14 + 16: 0, 2 * 16 + 15 + 16: 1}  # sequence 2: positions 30, 31 on page 3; 32 is past the table
    for t, t0 in ((c.k, before[0]), (c.v, before[1])):
        changed = (t != t0).flatten(1).any(1).cpu().numpy()
        assert list(np.nonzero(changed)[0]) == sorted(new)
    assert torch.equal(c.v[62], x[2, 0]) and torch.equal(c.v[63], x[2, 1])


# ---- gather ---------------------------------------------------------------------


@pytest.mark.parametrize("kind", [BF, F32, F8])
@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("D,Hkv,page", [(64, 1, 16), (128, 3, 64), (64, 8, 32)])
def test_gather(kind, dt, D, Hkv, page):
    rng = np.random.default_rng(D + Hkv)
    lens, starts = [0, 37, 0, 1, 130, 0], [3, 0, 7, 200, 11, 0]
    pages, n_pages = R.page_table(rng, [a + b for a, b in zip(lens, starts)], page)
    c = make_cache(rng, n_pages, page, Hkv, D, kind)
    cu = 2 + np.concatenate([[0], np.cumsum(lens)])   # two rows before the first, three behind the last
    n = int(cu[-1]) + 3
    out = [torch.full((n, Hkv, D), 9.0, dtype=dt, device=DEV) for _ in range(2)]
    c.gather(dev(pages), dev(cu), n, starts=dev(starts), out=out)
    for name, g in zip("kv", out):
        all_rows = torch.as_tensor(held(c, name))
        want = torch.full((n, Hkv, D), 9.0, dtype=torch.float64)
        for b, m in enumerate(lens):
            want[cu[b]:cu[b] + m] = all_rows[R.rows_of(pages, b, range(starts[b], starts[b] + m), page)]
        assert torch.equal(g.cpu().double(), want.to(dt).double())  # one rounding, or none


def test_gather_many_sequences_and_bad_pages():
    rng = np.random.default_rng(3)
    B, page = 150, 16
    lens = rng.integers(0, 40, B)
    lens[70:140] = 0
    pages, n_pages = R.page_table(rng, list(lens), page)
    pages[5, 1], pages[6, 0] = n_pages, -7
    lens[5], lens[6] = 20, 3
    c = make_cache(rng, n_pages, page, 2, 64, BF)
    cu = np.concatenate([[0], np.cumsum(lens)])
    k, v = c.gather(dev(pages), dev(cu), int(cu[-1]), max_len=pages.shape[1] * page)
    for g, name in ((k, "k"), (v, "v")):
        src = torch.as_tensor(held(c, name))
        for b in range(B):
            got = g[cu[b]:cu[b + 1]].cpu().double()
            for p in range(lens[b]):
                pg = pages[b, p // page]
                if 0 <= pg < n_pages:
                    assert torch.equal(got[p], src[pg * page + p % page])
                else:
                    assert torch.isnan(got[p]).all()


# ---- attend ---------------------------------------------------------------------


def run_attend(rng, dt, kind, D, Hq, Hkv, lens, T, page, mask="random", counts=None, qscale=2.0, stride=0,
               spoil=None, max_len=None):
    B = len(lens)
    counts_ = np.full(B, T) if counts is None else np.asarray(counts)
    pages, n_pages = R.page_table(rng, [p + T for p in lens], page)
    c = make_cache(rng, n_pages, page, Hkv, D, kind)
    m = {"random": lambda: R.random_tree(rng, B, T), "causal": lambda: None,
         "sparse": lambda: ((rng.random((B, T, T)) < 0.15) & (np.arange(T) % 4 != 1)[:, None]).astype(np.uint8) * 3}[mask]()
    q = torch.as_tensor(rng.standard_normal((B, T, Hq * D + stride)) * qscale, dtype=F32).to(dt).to(DEV)
    q = q[..., :Hq * D].unflatten(2, (Hq, D))
    if spoil:
        spoil(c, pages, m)
    out = torch.full((B, T, Hq, D), 5.0, dtype=dt, device=DEV)
    got = c.attend(dev(pages), dev(lens), q, mask=None if m is None else dev(m, torch.uint8),
                   counts=None if counts is None else dev(counts), out=out, max_len=max_len)
    assert got is out
    k, v = held(c, "k"), held(c, "v")
    with np.errstate(invalid="ignore"):
        want, wt, sc = R.attend(f64(q), k, v, pages, page, lens, counts_, m, D ** -0.5)
    tol = R.tolerance(dt, D, max(lens) + T, want, wt, sc)
    g = f64(out)
    for b in range(B):
        n = counts_[b]
        err = np.abs(g[b, :n] - want[b, :n])
        assert np.all(err <= tol[b, :n]), (b, float((err / tol[b, :n]).max()))
        assert np.all(g[b, n:] == 5.0)
    return c, pages, q, out, m


TYPES = [(BF, BF), (BF, F8), (F32, F32), (F32, F8)]


@pytest.mark.parametrize("dt,kind", TYPES)
@pytest.mark.parametrize("D,Hq,Hkv", [(64, 4, 4), (128, 4, 1), (128, 6, 2), (64, 7, 1), (128, 8, 1)])
@pytest.mark.parametrize("T", [1, 9, 33])
def test_attend_trees(dt, kind, D, Hq, Hkv, T):
    rng = np.random.default_rng(T + D + Hq)
    run_attend(rng, dt, kind, D, Hq, Hkv, [0, 1, 63, 200, 130], T, 16)


@pytest.mark.parametrize("dt,kind", TYPES)
def test_attend_lengths_around_tiles(dt, kind):
    """Prefixes that end on, before and behind tile and page borders."""
    rng = np.random.default_rng(7)
    run_attend(rng, dt, kind, 64, 2, 2, [31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257], 5, 32)


@pytest.mark.parametrize("dt,kind", TYPES)
@pytest.mark.parametrize("mask", ["causal", "random"])
def test_attend_many_rows(dt, kind, mask):
    """More rows than a tile takes, some sequences shorter than the batch's nodes."""
    rng = np.random.default_rng(8)
    run_attend(rng, dt, kind, 64, 4, 1, [70, 0, 300], 75, 64, mask=mask, counts=[75, 40, 0])


def test_attend_chunk_causal():
    rng = np.random.default_rng(9)
    run_attend(rng, BF, BF, 128, 2, 1, [100], 300, 128, mask="causal")


def test_attend_long_history():
    """One token behind a history that many workgroups share."""
    rng = np.random.default_rng(10)
    run_attend(rng, BF, F8, 128, 4, 2, [9000, 3], 1, 64, mask="causal")
    run_attend(rng, F32, F32, 64, 2, 1, [5000], 2, 16, mask="causal")


def test_attend_rows_that_see_nothing():
    """Sparse masks (not trees; rows empty, nodes not seeing themselves): with no
    prefix an empty row is zero."""
    rng = np.random.default_rng(11)
    for dt, kind in TYPES:
        _, _, _, out, m = run_attend(rng, dt, kind, 64, 2, 1, [0, 40], 12, 16, mask="sparse")
        empty = ~(m[0] != 0).any(-1)
        assert empty.sum() >= 3 and np.all(f64(out)[0][empty] == 0)


@pytest.mark.parametrize("dt,kind", TYPES)
@pytest.mark.parametrize("T,Hq", [(6, 2), (70, 4)])
def test_attend_masked_places_never_matter(dt, kind, T, Hq):
    """NaN and infinities in the keys and values of nodes that only some nodes see:
    the others' results are as without; those that see them get NaN or infinity."""
    rng = np.random.default_rng(12)
    page, lens, D = 16, [0, 21], 64
    B = len(lens)
    pages, n_pages = R.page_table(rng, [p + T for p in lens], page)
    c = make_cache(rng, n_pages, page, 1, D, kind)
    m = R.random_tree(rng, B, T)
    bad = T - 3   # a node that few others descend from
    q = torch.as_tensor(rng.standard_normal((B, T, Hq, D)), dtype=F32).to(dt).to(DEV)
    args = dict(mask=dev(m, torch.uint8))
    for b in range(B):
        row = R.rows_of(pages, b, [lens[b] + bad], page)[0]
        nan = 127 if kind == F8 else float("nan")
        inf = 127 if kind == F8 else float("inf")
        kk, vv = (c.k.view(torch.uint8), c.v.view(torch.uint8)) if kind == F8 else (c.k, c.v)
        kk[row, 0, 3], kk[row, 0, 5] = nan, inf
        vv[row, 0, 7], vv[row, 0, 9] = nan, inf
    got = f64(c.attend(dev(pages), dev(lens), q, **args))
    with np.errstate(invalid="ignore"):
        want, wt, sc = R.attend(f64(q), held(c, "k"), held(c, "v"), pages, page, lens, [T] * B, m, D ** -0.5)
    tol = R.tolerance(dt, D, max(lens) + T, want, wt, sc)
    for b in range(B):
        sees = m[b, :, bad] != 0
        assert sees.any() and not sees.all()
        assert np.all(np.abs(got[b] - want[b])[~sees] <= tol[b][~sees])
        assert np.isnan(got[b][sees]).all()
    # values alone: only their dims are touched, an infinity stays one
    for b in range(B):
        row = R.rows_of(pages, b, [lens[b] + bad], page)[0]
        kk[row] = 0
    got = f64(c.attend(dev(pages), dev(lens), q, **args))
    for b in range(B):
        sees = m[b, :, bad] != 0
        assert np.isnan(got[b][sees][..., 7]).all()
        assert np.all(np.isnan(got[b][sees][..., 9]) if kind == F8 else got[b][sees][..., 9] == np.inf)
        rest = [d for d in range(D) if d not in (7, 9)]
        assert np.isfinite(got[b][sees][..., rest]).all() and np.isfinite(got[b][~sees]).all()


def test_attend_reads_nothing_past_the_end():
    """Rows behind a sequence's nodes (rest of the page, other pages) hold NaN."""
    rng = np.random.default_rng(13)

    def spoil(c, pages, m):
        live = set()
        for b, p in enumerate([17, 64]):
            live |= set(R.rows_of(pages, b, range(p + 3), 16))
        rest = [r for r in range(c.k.shape[0]) if r not in live]
        c.k[rest] = float("nan")
        c.v[rest] = float("nan")
    run_attend(rng, BF, BF, 64, 4, 2, [17, 64], 7, 16, counts=[3, 3], spoil=spoil)


def test_attend_strided_queries_and_bound():
    rng = np.random.default_rng(14)
    run_attend(rng, BF, BF, 128, 4, 2, [50, 10], 6, 32, stride=64)
    run_attend(rng, F32, F32, 64, 4, 2, [50, 10], 6, 32, stride=4, max_len=56)


@pytest.mark.parametrize("dt,kind", TYPES)
def test_attend_bad_lengths_and_pages(dt, kind):
    """Sequences whose lengths or pages do not fit become NaN, the others stay."""
    rng = np.random.default_rng(15)
    B, T, D, page, Hq = 7, 3, 64, 16, 2
    pages, n_pages = R.page_table(rng, [40 + T] * B, page)
    c = make_cache(rng, n_pages, page, 1, D, kind)
    q = torch.as_tensor(rng.standard_normal((B, T, Hq, D)), dtype=F32).to(dt).to(DEV)
    lens = np.array([40, -1, 46, 40, 40, 40, 2 ** 31 - 2])
    counts = np.array([3, 3, 3, -2, 3, 4, 3])
    pages[4, 1] = n_pages + 3
    out = torch.full((B, T, Hq, D), 5.0, dtype=dt, device=DEV)
    c.attend(dev(pages), dev(lens), q, counts=dev(counts), out=out)
    g = f64(out)
    want, wt, sc = R.attend(f64(q)[:1], held(c, "k"), held(c, "v"), pages, page, lens[:1], counts[:1], None, D ** -0.5)
    assert np.all(np.abs(g[0] - want[0]) <= R.tolerance(dt, D, 43, want, wt, sc)[0])
    assert np.isnan(g[1:]).all()


def test_attend_is_deterministic_and_captured():
    """The same bits every time, eagerly on another stream and replayed from a graph
    while eager work goes on."""
    rng = np.random.default_rng(16)
    B, T, Hq, Hkv, D, page = 5, 17, 8, 2, 128, 64
    lens = [900, 3, 0, 411, 1500]
    pages, n_pages = R.page_table(rng, [p + T for p in lens], page)
    c = make_cache(rng, n_pages, page, Hkv, D, F8)
    q = torch.as_tensor(rng.standard_normal((B, T, Hq, D)), dtype=F32).to(BF).to(DEV)
    pg, ln, m = dev(pages), dev(lens), dev(R.random_tree(rng, B, T), torch.uint8)
    want = c.attend(pg, ln, q, mask=m).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = c.attend(pg, ln, q, mask=m)
    side.synchronize()
    assert torch.equal(want, other)
    ws = [c.attend_workspace(B, T, Hq, pages.shape[1] * page) for _ in range(2)]
    outs = [torch.empty_like(q) for _ in range(2)]
    q2 = q.flip(0).contiguous()
    want2 = c.attend(pg, ln, q2, mask=m).clone()
    graphs = []
    torch.cuda.synchronize()
    for i, x in enumerate((q, q2)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.attend(pg, ln, x, mask=m, out=outs[i], workspace=ws[i])
        graphs.append(g)
    for _ in range(4):
        for o in outs:
            o.zero_()
        for g in graphs:
            g.replay()
        eager = c.attend(pg, ln, q, mask=m)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want2) and torch.equal(eager, want)
    ln.copy_(dev([10, 20, 30, 40, 50]))   # the lengths are read when the graph runs
    for g in graphs:
        g.replay()
    assert torch.equal(outs[0], c.attend(pg, ln, q, mask=m))


def test_attend_offsets_past_32_bits():
    """A pool of more than 2^32 bytes per tensor, the sequence in its last pages."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    from paper_2509_20416_amd import PagedCache
    page, Hkv, D, n_pages = 1024, 8, 128, 2200   # 2.3 M rows, 4.6 GB in bf16
    c = PagedCache.empty(n_pages, page, Hkv, D, BF, DEV)
    rng = np.random.default_rng(17)
    pages = np.array([[n_pages - 1, n_pages - 2]])
    rows = slice((n_pages - 2) * page, n_pages * page)
    for t in (c.k, c.v):
        t[rows] = torch.as_tensor(rng.standard_normal((2 * page, Hkv, D)), dtype=F32).to(BF).to(DEV)
    small = PagedCache(c.k[rows].clone(), c.v[rows].clone(), page)
    q = torch.randn(1, 3, 16, D, device=DEV, dtype=BF)
    x = torch.randn(1, 3, Hkv, D, device=DEV, dtype=BF)
    near = dev([[1, 0]])
    for cache, pg in ((c, dev(pages)), (small, near)):
        cache.append(pg, dev([1500]), x, x)
    a = c.attend(dev(pages), dev([1500]), q)
    assert torch.equal(a, small.attend(near, dev([1500]), q))
    g = c.gather(dev(pages), dev([0, 1503]), 1503)
    w = small.gather(near, dev([0, 1503]), 1503)
    assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1])


# ---- commit ---------------------------------------------------------------------


@pytest.mark.parametrize("kind,layers,D", [(BF, 3, 64), (F8, 70, 64), (F32, 1, 128)])
def test_commit(kind, layers, D):
    """Paths whose rows are both source and destination (k = 2 < levels), any
    accepted length, more layers than one launch takes."""
    from paper_2509_20416_amd import commit_accepted
    rng = np.random.default_rng(layers)
    B, levels, topk, page, Hkv = 8, 6, 2, 16, 3
    T = 1 + levels * topk
    _, _, ret, _ = R.backbone(B, levels, topk)
    lens = rng.integers(0, 60, B)
    pages, n_pages = R.page_table(rng, [p + T for p in lens], page)
    caches = [make_cache(rng, n_pages, page, Hkv, D, kind) for _ in range(layers)]
    before = [(held(c, "k"), held(c, "v")) for c in caches]
    acc = np.array([0, 1, 2, 3, 4, 5, 6, 6])
    path = np.array([next(j for j in range(ret.shape[1]) if ret[b, j, acc[b]] >= 0) if b % 2 else
                     max(j for j in range(ret.shape[1]) if ret[b, j, acc[b]] >= 0) for b in range(B)])
    new = commit_accepted(caches, dev(pages), dev(lens), dev(ret), dev(path), dev(acc), nodes=T)
    assert new.tolist() == list(lens + 1 + acc)
    for c, (k0, v0) in zip(caches, before):
        wk, wv = k0.copy(), v0.copy()
        for b in range(B):
            for t in range(1, acc[b] + 1):
                d, s = (R.rows_of(pages, b, [lens[b] + x], page)[0] for x in (t, int(ret[b, path[b], t])))
                wk[d], wv[d] = k0[s], v0[s]
        assert np.array_equal(held(c, "k"), wk) and np.array_equal(held(c, "v"), wv)


def test_commit_leaves_bad_sequences():
    from paper_2509_20416_amd import commit_accepted
    rng = np.random.default_rng(2)
    B, levels, topk, page = 9, 3, 4, 16
    T = 1 + levels * topk
    _, _, ret, _ = R.backbone(B, levels, topk)
    lens = np.array([5, 5, 5, 5, -3, 5, 5, 40, 5])
    pages, n_pages = R.page_table(rng, [30] * B, page)
    acc = np.array([2, 4, -1, 2, 2, 2, 2, 2, 1])
    full = next(j for j in range(ret.shape[1]) if ret[0, j, levels] >= 0)   # a path to the last level
    path = np.full(B, full)
    path[3] = 99
    ret[5, full, 2], ret[6, full, 1] = T, -1
    pages[8, 0] = n_pages
    c = make_cache(rng, n_pages, page, 1, 64, BF)
    k0 = c.k.clone()
    new = commit_accepted([c], dev(pages), dev(lens), dev(ret), dev(path), dev(acc), nodes=T)
    assert new.tolist() == [8] + [-1] * 8
    want = k0.clone()
    for t in (1, 2):
        d, s = (R.rows_of(pages, 0, [5 + x], page)[0] for x in (t, int(ret[0, full, t])))
        want[d] = k0[s]
    assert torch.equal(c.k, want)


# ---- together -------------------------------------------------------------------


@pytest.mark.parametrize("kind", [BF, F8])
def test_cycles_of_one_layer(kind):
    """Prompt, then cycles of tree, attention, acceptance and commit through the
    drafter's own tree and acceptance: in the end the cache holds, position by
    position, what appending the emitted tokens one after the other holds, and the
    nodes on the accepted path saw exactly those."""
    from fe_synth import configs as CF, make_inputs, make_weights
    from paper_2509_20416_amd import Drafter, PagedCache, Rope, commit_accepted, fe
    cfg = CF.SMALL_GQA_BF16.with_(batch=3, prefix=40)
    B, N, k = 3, cfg.n_layers, cfg.topk
    T, Hq, Hkv, D, page = 1 + N * k, 4, 2, 64, 16
    dr = Drafter(cfg, make_weights(cfg, seed=1), device=DEV)
    rng = np.random.default_rng(4)
    vocab = cfg.target_vocab
    table = torch.as_tensor(rng.standard_normal((vocab, (Hq + 2 * Hkv) * D)), dtype=F32).to(BF).to(DEV)
    freqs, _ = fe.fe_rope_frequencies(D, 10000.0)
    rope = Rope(dev(freqs, torch.float64))
    pages, n_pages = R.page_table(rng, [120] * B, page)
    pg = dev(pages)
    c, plain = (make_cache(np.random.default_rng(9), n_pages, page, Hkv, D, kind) for _ in range(2))

    def parts(tokens):   # a stand-in for the target: what its projection gives depends on the token alone
        x = table[tokens.long()].unflatten(2, (Hq + 2 * Hkv, D))
        return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    seqs = [list(rng.integers(0, vocab, n)) for n in (7, 40, 21)]
    lens = dev([len(s) for s in seqs])
    pad = np.zeros((B, 40), np.int32)
    for b, s in enumerate(seqs):
        pad[b, :len(s)] = s
    q, kk, vv = parts(dev(pad))
    zero = dev([0] * B)
    q = c.append(pg, zero, kk, vv, counts=lens, rope=rope, q=q)
    c.attend(pg, zero, q, counts=lens)
    root = dev(rng.integers(0, vocab, B))
    inp = make_inputs(cfg, seed=3, prefix_lens=np.array([40] * B, np.int32))
    for cycle in range(4):
        di = dr.upload_inputs(inp)
        di.next_tokens.copy_(root)
        di.prefix_lens = lens
        tree = dr.build_tree(di, dr.forward(di)["topk_ids"])
        q, kk, vv = parts(tree["tokens"])
        q = c.append(pg, lens, kk, vv, positions=tree["positions"], rope=rope, q=q)
        out = c.attend(pg, lens, q, mask=tree["mask"])
        # the "target" agrees with a given path of the tree, then goes its own way
        ret, tok = tree["retrieve"].cpu().numpy(), tree["tokens"].cpu().numpy()
        nxt = rng.integers(0, vocab, (B, T)).astype(np.int32)
        for b in range(B):
            j = rng.integers(ret.shape[1])
            nodes = [x for x in ret[b, j] if x >= 0][:1 + int(rng.integers(0, N + 1))]
            for a, z in zip(nodes, nodes[1:]):
                nxt[b, a] = tok[b, z]
        acc = dr.accept_greedy(tree, dev(nxt))
        new = commit_accepted([c], pg, lens, tree["retrieve"], acc["accept_path"], acc["accept_len"], nodes=T)
        al, ap = acc["accept_len"].tolist(), acc["accept_path"].tolist()
        old = lens.tolist()
        for b in range(B):
            path = ret[b, ap[b], :al[b] + 1]
            seqs[b] += [int(tok[b, x]) for x in path]
            assert new[b].item() == len(seqs[b]) == old[b] + 1 + al[b]
        # the emitted tokens one after the other
        for b in range(B):
            s = dev(np.asarray(seqs[b])[None])
            q1, k1, v1 = parts(s)
            q1 = plain.append(pg[b:b + 1], dev([0]), k1, v1, rope=rope, q=q1)
            o1 = plain.attend(pg[b:b + 1], dev([0]), q1)
            rows = R.rows_of(pages, b, range(len(seqs[b])), page)
            assert torch.equal(c.k.view(torch.uint8)[rows], plain.k.view(torch.uint8)[rows])
            assert torch.equal(c.v.view(torch.uint8)[rows], plain.v.view(torch.uint8)[rows])
            path = ret[b, ap[b], :al[b] + 1]
            a, z = f64(out)[b, path], f64(o1)[0, old[b]:]
            # two bf16 results of one sum: both within 2^-8 (|v| weighted + |out|) of it, |v| < 5
            assert np.all(np.abs(a - z) <= 2 * 2.0 ** -8 * (5 + 2 * np.abs(z)))
        lens, root = new, dev([acc["accepted"][b, al[b]].item() for b in range(B)])
    cu = dev(np.concatenate([[0], np.cumsum([len(s) for s in seqs])]))
    n = int(cu[-1])
    for x, y in zip(c.gather(pg, cu, n), plain.gather(pg, cu, n)):
        assert torch.equal(x, y)
    dr.close()
