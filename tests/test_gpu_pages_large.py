"""pages_resize with counts next to 2^31: the numbers of a thread's elements must
not wrap behind the last one."""
import ctypes

import pytest
import torch

from gpu_util import Q

pytestmark = pytest.mark.gpu


def _put(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("capacity", [2**31 - 1, 2**31 - 2**19 + 5])
def test_token_capacity_next_to_2_31(capacity):
    """Slots of 35 new tokens, and -1 in every entry behind them."""
    P, old, new = 16, (20, 0, 40), (25, 30, 8)
    lens, want = _put(*old), _put(*new)
    table = torch.full((3, 8), -1, dtype=torch.int32, device="cuda")
    table[0, :2], table[2, :3] = _put(4, 5), _put(6, 7, 8)
    stack, count = _put(0, 1, 2, 3, -1, -1, -1, -1, -1), _put(4)
    small = [t.clone() for t in (lens, table, stack, count)]
    slots = torch.zeros(capacity, dtype=torch.int32, device="cuda")
    cu, status = torch.zeros(4, dtype=torch.int32, device="cuda"), _put(9)
    ws = torch.zeros(Q.lib().qnn_pages_workspace_size(3), dtype=torch.uint8, device="cuda")
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    Q._check(Q.lib().qnn_pages_resize(Q._stream(), 3, P, p(lens), p(want), p(table), 8, 8, p(stack), 9, p(count), p(cu), p(slots),
                                      None, capacity, p(status), p(ws)))
    torch.cuda.synchronize()
    few = Q.pages_resize(small[0], want, small[1], small[2], small[3], P, 64)
    assert int(status) == 0 and torch.equal(cu, few[0]) and torch.equal(slots[:64], few[1])
    for a, b in zip((lens, table, stack, count), small):
        assert torch.equal(a, b)
    assert int(slots[64:].max()) == -1 and int(slots[64:].min()) == -1
