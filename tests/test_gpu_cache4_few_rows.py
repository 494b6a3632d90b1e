"""The binding's checks of strides say nothing of rows that aren't there: tensors
without tokens, and one token out of a wider tensor of any row stride."""
import numpy as np
import pytest
import torch

from gpu_util import Q

pytestmark = pytest.mark.gpu


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def test_no_tokens():
    c = Q.Cache4(2, 16, 2, 64)
    none = torch.empty(0, dtype=torch.float16, device="cuda")
    for stride in ((1, 1, 1), (0, 0, 0), (128, 64, 1)):
        q, k = none.as_strided((0, 8, 64), stride), none.as_strided((0, 2, 64), stride)
        Q.cache4_append(c, k, k, _ints())
        assert Q.attention4(q, c, _ints(0).view(1, 1), _ints(5), cu_q=_ints(0, 0), max_q=1).shape == (0, 8, 64)
        assert Q.attention4(q, c, _ints().view(0, 1), _ints()).shape == (0, 8, 64)
    rk, rv = Q.cache4_read(c, _ints())
    assert rk.shape == rv.shape == (0, 2, 64)


def test_one_token_of_any_stride():
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.normal(size=(3, 1, 4, 64))).half().cuda()
    c, d = (Q.Cache4(1, 16, 4, 64, data=torch.zeros(1, 4 * 16 * 72, dtype=torch.uint8, device="cuda")) for _ in range(2))
    slot, table, ctx = _ints(3), _ints(0).view(1, 1), _ints(4)
    Q.cache4_append(c, x[0], x[1], slot)
    q, k, v = (t.as_strided((1, 4, 64), (257, 64, 1), t.storage_offset()) for t in x)
    Q.cache4_append(d, q, k, slot)
    torch.cuda.synchronize()
    assert torch.equal(c.data, d.data)
    out = torch.empty(1, 4, 64, dtype=torch.float16, device="cuda")
    y = Q.attention4(v, d, table, ctx, out=out.as_strided((1, 4, 64), (301, 64, 1)))
    assert torch.equal(y, Q.attention4(x[2], c, table, ctx))
