"""GPU parity of tree attention where its launch changes: row counts around every
tile, short and long bounds on the lengths, more sequences than a workgroup counts
at once, and enough keys that a workgroup's share runs over several sequences."""
import numpy as np
import pytest
import torch

from tests import paged_ref as R
from tests import test_gpu_paged as P

pytestmark = pytest.mark.gpu
BF, F32, F8 = P.BF, P.F32, P.F8


def check(rng, dt, kind, D, Hq, Hkv, lens, T, page, width=0, mask=None, counts=None, good=None):
    """One call against the reference; the table is `width` pages wide, of which only
    those that hold positions are valid.  `good`: the sequences to compare (the rest
    has to be NaN)."""
    B = len(lens)
    fits = [p if good is None or b in good else 40 for b, p in enumerate(lens)]
    pages, n_pages = R.page_table(rng, [p + T for p in fits], page)
    if width > pages.shape[1]:
        pages = np.concatenate([pages, np.full((B, width - pages.shape[1]), -7, np.int32)], 1)
    c = P.make_cache(rng, n_pages, page, Hkv, D, kind)
    q = torch.as_tensor(rng.standard_normal((B, T, Hq, D)) * 2, dtype=F32).to(dt).to(P.DEV)
    out = torch.full((B, T, Hq, D), 5.0, dtype=dt, device=P.DEV)
    c.attend(P.dev(pages), P.dev(lens), q, mask=None if mask is None else P.dev(mask, torch.uint8),
             counts=None if counts is None else P.dev(counts), out=out)
    counts = np.full(B, T) if counts is None else np.asarray(counts)
    some = np.arange(B) if good is None else np.array(sorted(good))
    lens, g = np.asarray(lens), P.f64(out)
    want, wt, sc = R.attend(P.f64(q)[some], P.held(c, "k"), P.held(c, "v"), pages[some], page, lens[some],
                            counts[some], None if mask is None else mask[some], D ** -0.5)
    tol = R.tolerance(dt, D, int(lens[some].max()) + T, want, wt, sc)
    for i, b in enumerate(some):
        n = counts[b]
        err = np.abs(g[b, :n] - want[i, :n])
        assert np.all(err <= tol[i, :n]), (b, float((err / tol[i, :n]).max()))
        assert np.all(g[b, n:] == 5.0)
    for b in set(range(B)) - set(some.tolist()):
        n = counts[b] if 0 <= counts[b] <= T else T
        assert np.isnan(g[b, :n]).all() and np.all(g[b, n:] == 5.0), b


@pytest.mark.parametrize("dt,kind", P.TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [16, 17, 32, 33, 128, 129, 256, 257])
@pytest.mark.parametrize("width", [0, 4096])
def test_row_counts_and_bounds(dt, kind, D, T, width):
    """T rows per KV head, with a bound near the lengths and one of 2^19."""
    rng = np.random.default_rng(T + D + width)
    check(rng, dt, kind, D, 2, 2, [37, 200], T, 128, width, R.random_tree(rng, 2, T))


@pytest.mark.parametrize("dt,kind", [(BF, BF), (BF, F8), (F32, F32)])
@pytest.mark.parametrize("B,T", [(300, 3), (700, 33)])
def test_more_sequences_than_threads(dt, kind, B, T):
    rng = np.random.default_rng(B)
    check(rng, dt, kind, 64, 2, 1, rng.integers(0, 60, B), T, 16, mask=R.random_tree(rng, B, T),
          counts=rng.integers(0, T + 1, B))


@pytest.mark.parametrize("dt,kind,Hq,Hkv,T,B,n", [(BF, BF, 64, 8, 17, 8, 5000), (BF, F8, 16, 16, 1, 16, 2500),
                                                 (F32, F32, 16, 16, 1, 16, 2500)])
def test_long_shares(dt, kind, Hq, Hkv, T, B, n):
    """A workgroup's share is more than 1024 keys and crosses segments."""
    rng = np.random.default_rng(n)
    check(rng, dt, kind, 64, Hq, Hkv, rng.integers(n - 300, n + 300, B), T, 64)


@pytest.mark.parametrize("dt,kind", P.TYPES)
def test_bad_lengths_between_long_ones(dt, kind):
    """Sequences that become NaN while every workgroup has several steps, so that a bad
    one may lie on the border of two."""
    rng = np.random.default_rng(4)
    B, T = 48, 40
    lens, counts = rng.integers(500, 900, B), rng.integers(1, T + 1, B)
    bad = [1, 7, 20, 33, 46, 47]
    lens[bad[:4]] = [-1, 2 ** 31 - 2, -2 ** 31, 1024]
    counts[bad[4:]] = [-2, T + 1]
    check(rng, dt, kind, 64, 4, 2, lens, T, 64, 16, counts=counts, good=set(range(B)) - set(bad))


@pytest.mark.parametrize("dt,kind", P.TYPES)
@pytest.mark.parametrize("T,Hq", [(200, 2), (130, 8)])
def test_masked_infinities_over_many_tiles(dt, kind, T, Hq):
    P.test_attend_masked_places_never_matter(dt, kind, T, Hq)
