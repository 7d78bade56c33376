"""Refusals of the paged-cache entry points, and the rotary frequencies: host code
only, no GPU (addresses are made up and never dereferenced)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def fe():
    from paper_2509_20416_amd import fe as _fe
    _fe.lib()
    return _fe


A = [(1 << 32) + (i << 28) for i in range(16)]   # addresses far apart


def cache(fe, **kw):
    v = dict(k=A[0], v=A[1], k_scale=A[2], v_scale=A[3], n_pages=64, page_rows=32, n_kv_heads=2, head_dim=64,
             dtype=fe.FE_F8)
    v.update(kw)
    return fe.fe_paged_kv(**v)


def table(fe, **kw):
    v = dict(pages=A[4], max_pages=8, max_len=256)
    v.update(kw)
    return fe.fe_page_table(**v)


BAD_CACHE = [
    (dict(dtype=3), "FE_E_INVALID"), (dict(n_pages=0), "FE_E_INVALID"), (dict(n_kv_heads=0), "FE_E_INVALID"),
    (dict(page_rows=0), "FE_E_INVALID"), (dict(page_rows=48), "FE_E_UNSUPPORTED"),
    (dict(page_rows=8), "FE_E_UNSUPPORTED"), (dict(page_rows=1 << 17), "FE_E_UNSUPPORTED"),
    (dict(n_kv_heads=257), "FE_E_UNSUPPORTED"), (dict(n_pages=1 << 26), "FE_E_UNSUPPORTED"), (dict(head_dim=96), "FE_E_UNSUPPORTED"),
    (dict(k=None), "FE_E_INVALID"), (dict(v=A[1] + 8), "FE_E_ALIGN"), (dict(k_scale=None), "FE_E_INVALID"),
    (dict(v_scale=A[3] + 2), "FE_E_ALIGN"),
]
BAD_TABLE = [
    (dict(pages=None), "FE_E_INVALID"), (dict(pages=A[4] + 1), "FE_E_ALIGN"), (dict(max_pages=0), "FE_E_INVALID"),
    (dict(max_len=0), "FE_E_INVALID"), (dict(max_len=257), "FE_E_INVALID"),
]


def append(fe, c=None, t=None, **kw):
    v = dict(batch=2, nodes=3, starts=A[5], counts=A[6], positions=A[7], rope=None, dtype=fe.FE_BF16, k=A[8],
             k_stride=128, v=A[9], v_stride=128, q=A[10], q_stride=256, n_q_heads=4, q_out=A[11], stream=0)
    v.update(kw)
    fe.fe_cache_append(c or cache(fe), t or table(fe), **v)


def gather(fe, c=None, t=None, **kw):
    v = dict(batch=2, starts=A[5], cu_rows=A[6], n_rows=9, dtype=fe.FE_BF16, k_out=A[7], v_out=A[8], stream=0)
    v.update(kw)
    fe.fe_cache_gather(c or cache(fe), t or table(fe), **v)


def attend(fe, c=None, t=None, **kw):
    v = dict(batch=2, nodes=3, n_q_heads=4, prefix_lens=A[5], counts=A[6], mask=A[7], dtype=fe.FE_BF16, q=A[8],
             q_stride=256, scale=0.125, out=A[9], workspace=A[10], ws_bytes=1 << 40, stream=0)
    v.update(kw)
    fe.fe_tree_attention(c or cache(fe), t or table(fe), **v)


def commit(fe, c=None, t=None, **kw):
    v = dict(batch=2, nodes=9, n_paths=4, depth=2, prefix_lens=A[5], retrieve=A[6], accept_path=A[7],
             accept_len=A[8], new_lens=A[9], stream=0)
    v.update(kw)
    cs = (fe.fe_paged_kv * 2)(c or cache(fe), c or cache(fe))
    fe.fe_cache_commit(kw.pop("caches", cs), v.pop("n_layers", 2), t or table(fe),
                       **{k: x for k, x in v.items() if k != "caches"})


@pytest.mark.parametrize("call", [append, gather, attend, commit])
def test_bad_caches_and_tables(fe, call):
    for kw, status in BAD_CACHE:
        with pytest.raises(fe.FeError, match=status):
            call(fe, c=cache(fe, **kw))
    for kw, status in BAD_TABLE:
        with pytest.raises(fe.FeError, match=status):
            call(fe, t=table(fe, **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), "FE_E_INVALID"), (dict(batch=65536), "FE_E_INVALID"), (dict(nodes=-1), "FE_E_INVALID"),
    (dict(nodes=1 << 30), "FE_E_INVALID"), (dict(dtype=2), "FE_E_INVALID"), (dict(k=None), "FE_E_INVALID"),
    (dict(k=A[8] + 8), "FE_E_ALIGN"), (dict(k_stride=127), "FE_E_INVALID"), (dict(v_stride=132), "FE_E_ALIGN"),
    (dict(v_stride=(1 << 31) + 8), "FE_E_INVALID"), (dict(q_out=None), "FE_E_INVALID"),
    (dict(q_out=A[11] + 4), "FE_E_ALIGN"), (dict(n_q_heads=0), "FE_E_INVALID"),
    (dict(n_q_heads=1025, q_stride=1 << 20), "FE_E_INVALID"), (dict(q_out=A[10] + 512), "FE_E_INVALID"),
    (dict(starts=None), "FE_E_INVALID"), (dict(counts=A[6] + 2), "FE_E_ALIGN"),
    (dict(positions=A[7] + 1), "FE_E_ALIGN"),
])
def test_append_refuses(fe, kw, status):
    with pytest.raises(fe.FeError, match=status):
        append(fe, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(freqs=None), "FE_E_INVALID"), (dict(freqs=A[12] + 4), "FE_E_ALIGN"), (dict(rotary_dim=0), "FE_E_INVALID"),
    (dict(rotary_dim=24), "FE_E_UNSUPPORTED"), (dict(rotary_dim=80), "FE_E_INVALID"), (dict(layout=2), "FE_E_INVALID"),
    (dict(magnitude=0.0), "FE_E_INVALID"), (dict(magnitude=math.inf), "FE_E_INVALID"),
    (dict(magnitude=math.nan), "FE_E_INVALID"),
])
def test_append_refuses_rope(fe, kw, status):
    v = dict(freqs=A[12], rotary_dim=64, layout=0, magnitude=1.0)
    v.update(kw)
    with pytest.raises(fe.FeError, match=status):
        append(fe, rope=fe.fe_rope(**v))


def test_type_pairs(fe):
    for held, dtype in ((fe.FE_BF16, fe.FE_F32), (fe.FE_F32, fe.FE_BF16)):
        for call in (append, attend):
            with pytest.raises(fe.FeError, match="FE_E_UNSUPPORTED"):
                call(fe, c=cache(fe, dtype=held), dtype=dtype)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-2), "FE_E_INVALID"), (dict(n_rows=-1), "FE_E_INVALID"), (dict(dtype=2), "FE_E_INVALID"),
    (dict(k_out=None, v_out=None), "FE_E_INVALID"), (dict(k_out=A[7] + 2), "FE_E_ALIGN"),
    (dict(cu_rows=None), "FE_E_INVALID"), (dict(cu_rows=A[6] + 2), "FE_E_ALIGN"), (dict(starts=A[5] + 1), "FE_E_ALIGN"),
])
def test_gather_refuses(fe, kw, status):
    with pytest.raises(fe.FeError, match=status):
        gather(fe, **kw)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=-1), "FE_E_INVALID"), (dict(nodes=-1), "FE_E_INVALID"), (dict(n_q_heads=3), "FE_E_INVALID"),
    (dict(n_q_heads=0), "FE_E_INVALID"), (dict(n_q_heads=1026, q_stride=1 << 20), "FE_E_UNSUPPORTED"),
    (dict(nodes=(1 << 19) + 1), "FE_E_UNSUPPORTED"), (dict(q=None), "FE_E_INVALID"), (dict(q=A[8] + 4), "FE_E_ALIGN"),
    (dict(q_stride=255), "FE_E_INVALID"), (dict(q_stride=260), "FE_E_ALIGN"), (dict(out=None), "FE_E_INVALID"),
    (dict(out=A[8]), "FE_E_INVALID"), (dict(prefix_lens=None), "FE_E_INVALID"),
    (dict(prefix_lens=A[5] + 2), "FE_E_ALIGN"), (dict(counts=A[6] + 1), "FE_E_ALIGN"), (dict(scale=0.0), "FE_E_INVALID"),
    (dict(scale=math.inf), "FE_E_INVALID"), (dict(workspace=None), "FE_E_WORKSPACE"), (dict(ws_bytes=16), "FE_E_WORKSPACE"),
    (dict(workspace=A[10] + 128), "FE_E_ALIGN"),
])
def test_attention_refuses(fe, kw, status):
    with pytest.raises(fe.FeError, match=status):
        attend(fe, **kw)


def test_attention_workspace_bytes(fe):
    args = (table(fe), 2, 3, 4, fe.FE_BF16)
    assert fe.fe_tree_attention_workspace_bytes(cache(fe), *args) > 0
    assert fe.fe_tree_attention_workspace_bytes(cache(fe, head_dim=32), *args) == 0
    assert "head_dim" in fe.fe_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(n_layers=0), "FE_E_INVALID"), (dict(n_layers=1025), "FE_E_INVALID"), (dict(nodes=0), "FE_E_INVALID"),
    (dict(n_paths=0), "FE_E_INVALID"), (dict(depth=-1), "FE_E_INVALID"), (dict(depth=17), "FE_E_UNSUPPORTED"),
    (dict(batch=-1), "FE_E_INVALID"), (dict(retrieve=None), "FE_E_INVALID"), (dict(new_lens=None), "FE_E_INVALID"),
    (dict(accept_len=A[8] + 1), "FE_E_ALIGN"), (dict(new_lens=A[5]), "FE_E_INVALID"),
    (dict(new_lens=A[8] + 4), "FE_E_INVALID"),
])
def test_commit_refuses(fe, kw, status):
    with pytest.raises(fe.FeError, match=status):
        commit(fe, **kw)


def test_commit_refuses_unlike_layers(fe):
    for kw in (dict(n_pages=63), dict(page_rows=64), dict(head_dim=128), dict(n_kv_heads=1), dict(dtype=fe.FE_BF16)):
        cs = (fe.fe_paged_kv * 2)(cache(fe), cache(fe, **kw))
        with pytest.raises(fe.FeError, match="FE_E_INVALID"):
            commit(fe, caches=cs)


def test_empty_calls_do_nothing(fe):
    append(fe, batch=0)
    append(fe, nodes=0)
    attend(fe, batch=0)
    attend(fe, nodes=0)
    gather(fe, n_rows=0)
    gather(fe, batch=0)
    commit(fe, batch=0)


# ---- frequencies ------------------------------------------------------------------


def test_frequencies(fe):
    R, theta = 96, 500000.0
    m = np.arange(R // 2)
    w = theta ** (-2.0 * m / R)
    got, mag = fe.fe_rope_frequencies(R, theta)
    np.testing.assert_allclose(got, w, rtol=1e-14)
    assert mag == 1.0
    got, mag = fe.fe_rope_frequencies(R, theta, fe.FE_SCALE_LINEAR, 8.0)
    np.testing.assert_allclose(got, w / 8, rtol=1e-14)
    got, mag = fe.fe_rope_frequencies(R, theta, fe.FE_SCALE_BANDED, 8.0, 1.0, 4.0, 8192.0)
    wave = 2 * math.pi / w
    assert mag == 1.0
    keep, slow = wave < 8192 / 4.0, wave > 8192 / 1.0
    np.testing.assert_allclose(got[keep], w[keep], rtol=1e-14)
    np.testing.assert_allclose(got[slow], w[slow] / 8, rtol=1e-14)
    mid = ~keep & ~slow
    s = (8192 / wave[mid] - 1.0) / 3.0
    np.testing.assert_allclose(got[mid], (1 - s) * w[mid] / 8 + s * w[mid], rtol=1e-12)
    assert keep.any() and slow.any() and mid.any()
    got, mag = fe.fe_rope_frequencies(R, 10000.0, fe.FE_SCALE_RAMP, 16.0, 1.0, 32.0, 4096.0)
    w = 10000.0 ** (-2.0 * m / R)
    assert abs(mag - (0.1 * math.log(16) + 1)) < 1e-7
    a = math.floor(R * math.log(4096 / (32 * 2 * math.pi)) / (2 * math.log(10000)))
    b = math.ceil(R * math.log(4096 / (1 * 2 * math.pi)) / (2 * math.log(10000)))
    r = np.clip((m - a) / (b - a), 0, 1)
    np.testing.assert_allclose(got, w / 16 * r + w * (1 - r), rtol=1e-12)
    assert 0 < a < b < R // 2


@pytest.mark.parametrize("a", [
    (0, 1e4), (7, 1e4), (64, 1.0), (64, math.inf), (64, 1e4, 4), (64, 1e4, 1, 0.5), (64, 1e4, 1, math.nan),
    (64, 1e4, 2, 8.0, 0.0, 4.0, 8192.0), (64, 1e4, 2, 8.0, 4.0, 4.0, 8192.0), (64, 1e4, 3, 8.0, 1.0, 32.0, 0.0),
])
def test_frequencies_refuse(fe, a):
    with pytest.raises(fe.FeError, match="FE_E_INVALID"):
        fe.fe_rope_frequencies(*a)


# ---- the tensors' side: refused before anything reaches the library --------------------


def test_tensor_checks(fe):
    from paper_2509_20416_amd import PagedCache, Rope, commit_accepted
    bf = torch.bfloat16
    k = torch.zeros(64, 2, 64, dtype=bf)
    c = PagedCache(k, k.clone(), 16)
    pages, i2 = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    x, q = torch.zeros(2, 3, 2, 64, dtype=bf), torch.zeros(2, 3, 4, 64, dtype=bf)

    def refused(f, *a, status="FE_E_INVALID", **kw):
        with pytest.raises(fe.FeError, match=status):
            f(*a, **kw)
    refused(PagedCache, k, k[:, :1].contiguous(), 16)
    refused(PagedCache, k, k.float(), 16)
    refused(PagedCache, k, k, 48)
    refused(PagedCache, k[:, ::2], k[:, ::2], 16)
    refused(PagedCache, k.half(), k.half(), 16, status="FE_E_UNSUPPORTED")
    refused(PagedCache, k.to(torch.uint8), k.to(torch.uint8), 16)
    refused(PagedCache, k.to(torch.uint8), k.to(torch.uint8), 16, torch.zeros(64, 2, dtype=torch.uint8),
            torch.zeros(64, 2, dtype=torch.uint8))
    refused(Rope, torch.zeros(32))
    refused(Rope, torch.zeros(32, dtype=torch.float64), "halves")
    refused(c.append, pages, i2, x, x.float())
    refused(c.append, pages, i2, x, x[:, :2])
    refused(c.append, pages, i2.long(), x, x)
    refused(c.append, pages, i2[:1], x, x)
    refused(c.append, pages[:1], i2, x, x)
    refused(c.append, pages, i2, x.transpose(1, 2).contiguous().transpose(1, 2), x)
    refused(c.append, pages, i2, x, x, q=q, q_out=q[:, :, :2])
    refused(c.append, pages, i2, x, x, positions=torch.zeros(2, 2, dtype=torch.int32))
    refused(c.append, pages, i2, x.half(), x.half(), status="FE_E_UNSUPPORTED")
    refused(c.gather, pages, i2, 4)
    refused(c.gather, pages, torch.zeros(3, dtype=torch.int32), 4, out=(k, k))
    refused(c.attend, pages, i2, q, mask=torch.zeros(2, 3, 3, dtype=torch.bool))
    refused(c.attend, pages, i2, q, mask=torch.zeros(2, 3, 2, dtype=torch.uint8))
    refused(c.attend, pages, i2, q, out=q.float())
    refused(c.attend, pages, i2, q[..., :32])
    refused(c.attend, pages, i2, q, counts=torch.zeros(3, dtype=torch.int32))
    ret = torch.zeros(2, 4, 3, dtype=torch.int32)
    refused(commit_accepted, [], pages, i2, ret, i2, i2, 9)
    refused(commit_accepted, [c], pages, i2, ret[0], i2, i2, 9)
    refused(commit_accepted, [c], pages, i2, ret, i2[:1], i2, 9)
    # and nothing on the host reaches a kernel
    refused(c.append, pages, i2, x, x, status="FE_E_UNSUPPORTED")
    refused(c.attend, pages, i2, q, status="FE_E_UNSUPPORTED")
    refused(c.gather, pages, torch.zeros(3, dtype=torch.int32), 4, status="FE_E_UNSUPPORTED")
    refused(commit_accepted, [c], pages, i2, ret, i2, i2, 9, status="FE_E_UNSUPPORTED")
