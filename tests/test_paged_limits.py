"""More refusals of the paged-cache entry points (host code only, no GPU)."""
import pytest

from tests import test_paged_abi as A
from tests.test_paged_abi import fe  # noqa: F401 (fixture)


def test_attention_refuses_too_many_keys(fe):
    c, t = A.cache(fe, n_kv_heads=128, n_pages=1 << 15, page_rows=32768), A.table(fe, max_pages=1 << 15, max_len=1 << 30)
    with pytest.raises(fe.FeError) as e:
        A.attend(fe, c, t, n_q_heads=128, q_stride=128 * 64)
    assert e.value.status == fe.FE_E_UNSUPPORTED
    assert fe.fe_tree_attention_workspace_bytes(c, t, 2, 3, 128, fe.FE_BF16) == 0
    t = A.table(fe, max_pages=1 << 15, max_len=1 << 29)
    assert fe.fe_tree_attention_workspace_bytes(c, t, 2, 3, 128, fe.FE_BF16) > 0


@pytest.mark.parametrize("kw", [dict(), dict(k=A.A[12]), dict(v=A.A[12])])
def test_commit_refuses_layers_that_share_a_cache(fe, kw):
    cs = (fe.fe_paged_kv * 3)(A.cache(fe), A.cache(fe, k=A.A[13], v=A.A[14]), A.cache(fe, **kw))
    with pytest.raises(fe.FeError) as e:
        A.commit(fe, caches=cs, n_layers=3)
    assert e.value.status == fe.FE_E_INVALID
