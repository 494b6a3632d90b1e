"""Numbers beyond 32 bits are refused by the cache's binding, not cut off."""
import pytest
import torch

from paper_2006_10226_amd import qnn as Q

WRAPS = (2**32 + 1, 2**31, -2**31 - 1)


@pytest.mark.parametrize("n", WRAPS)
def test_plain_numbers(n):
    Q.lib()
    with pytest.raises(ValueError, match="32 bits"):
        Q._one_q(0.1, n)
    for k in range(4):
        a = [3, 16, 2, 64]
        a[k] = n
        with pytest.raises(ValueError, match="32 bits"):
            Q.Cache4(*a, data=torch.zeros(1))


@pytest.mark.gpu
@pytest.mark.parametrize("n", WRAPS)
def test_calls(n):
    put = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    c = Q.Cache4(2, 16, 2, 64)
    q = torch.zeros(1, 4, 64, dtype=torch.float16, device="cuda")
    for name in ("max_q", "max_ctx", "window"):
        with pytest.raises(ValueError, match="32 bits"):
            Q.attention4(q, c, put(0).view(1, 1), put(1), put(0, 1), **{name: n})
        with pytest.raises(ValueError, match="32 bits"):
            Q.attention4_workspace_size(c, 1, 4, 1, 1, **{name: n})
    with pytest.raises(ValueError, match="32 bits"):
        Q.attention4(q.to(torch.int8), c, put(0).view(1, 1), put(1), q_zp=n)
    for kw in (dict(page_size=n, token_capacity=4), dict(page_size=16, token_capacity=n)):
        with pytest.raises(ValueError):
            Q.pages_resize(put(0), put(1), put(-1).view(1, 1), put(0), put(1), **kw)
