"""Calls of more threads than a launch takes (2^32) are refused by the cache's
entry points before any device work (no GPU needed)."""
import pytest

from test_cache4_cpu import Q, _append, _attend, _cache, _read  # noqa: F401


# 256 threads for 16, 8, 4 tokens of a head (DP 64, 128, 256)
@pytest.mark.parametrize("dim,heads,tokens", [(64, 1, 2**28), (64, 4096, 2**16), (72, 2, 2**26), (128, 16, 2**23 - 7),
                                              (256, 8, 2**23), (136, 4096, 2**14), (64, 2, 2**31 - 1)])
def test_append_and_read(Q, dim, heads, tokens):  # noqa: F811
    c = _cache(Q, heads=heads, head_dim=dim)
    ld = heads * dim
    for st, msg in (_append(Q, c, tokens=tokens, k_ld=ld, v_ld=ld), _read(Q, c, tokens=tokens, k_ld=ld, v_ld=ld)):
        assert st == "QNN_ERR_UNSUPPORTED" and msg


# rows of max_q queries by two query heads a cache head (two cache heads)
@pytest.mark.parametrize("kw", [dict(requests=1024, max_q=2**18, tokens=2**20), dict(requests=2**18, max_q=1024, tokens=2**20),
                                dict(requests=2**23, max_q=1, tokens=2**23), dict(requests=1, max_q=2**28, tokens=2**28)])
def test_attention(Q, kw):  # noqa: F811
    st, msg = _attend(Q, **kw)
    assert st == "QNN_ERR_UNSUPPORTED" and msg


def test_sizes_that_no_sum_holds(Q):  # noqa: F811
    """Products of the sizes beyond 64 bits: refused, and no workspace."""
    for heads, q_heads in ((1, 2**20), (1, 2**31 - 1), (4096, 2**30)):
        c = _cache(Q, heads=heads)
        for requests, max_q in ((2**30, 2**30), (2**31 - 1, 2**31 - 1), (2**21, 2**30)):
            ld = q_heads * 64
            p = Q.AttentionParams(2**12, q_heads, requests, 8, ld, ld, 8, max_q, 0, 1, 0, 0.1)
            assert Q.lib().qnn_attention4_workspace_size(c, p) == 0
            st, msg = _attend(Q, c, tokens=2**12, q_heads=q_heads, requests=requests, q_ld=ld, o_ld=ld, max_q=max_q)
            assert st == "QNN_ERR_UNSUPPORTED" and msg


def test_max_q_counts_for_nothing_without_cu(Q):  # noqa: F811
    """One query a request: the workspace is the same whatever max_q says."""
    p = [Q.AttentionParams(2, 4, 2, 4096, 256, 256, 4096, most, 0, 1, 0, 0.1) for most in (1, 2**31 - 1)]
    size = [Q.lib().qnn_attention4_workspace_size(_cache(Q, page_size=64), v) for v in p]
    assert size[0] == size[1] > 0
