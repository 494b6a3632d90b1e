"""attention4 with cu_q and without max_q computes every query."""
import pytest
import torch

from gpu_util import Q
from test_gpu_attention4 import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(ctx=[40, 33, 7], nq=[12, 1, 7]), dict(ctx=[2500, 90], nq=[1, 40]), dict(ctx=[3000, 64], nq=[1, 1]),
                                dict(ctx=[5], nq=[0])])
def test_every_query_is_computed(kw):
    c = Case(128, 16, 2, 4, **kw)
    a = c.device()
    del a["max_q"]
    out = torch.full(tuple(c.q.shape), float("nan"), dtype=torch.float16, device="cuda")
    c.check(Q.attention4(**a, out=out), "no max_q")
    # a workspace of the size for these defaults serves
    T, Hq, _ = c.q.shape
    size = Q.attention4_workspace_size(c.c, T, Hq, len(c.ctx), c.W, max_ctx=a["max_ctx"])
    out.fill_(float("nan"))
    c.check(Q.attention4(**a, out=out, workspace=torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")), "workspace")


def test_too_many_for_a_grid_is_said():
    c = Case(64, 16, 1, 1, ctx=[3] * 4096, nq=[1] * 4096)
    a = c.device()
    del a["max_q"]
    T = 2**18   # 4096 requests of up to 2^18 queries
    a["q"] = torch.zeros(T, 1, 64, dtype=torch.float16, device="cuda")
    with pytest.raises(Q.QnnError, match="UNSUPPORTED"):
        Q.attention4(**a)
