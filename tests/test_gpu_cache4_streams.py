"""cache4_append refuses a stream of another device than the cache's, as the calls
that allocate do by making the stream's device the current one."""
import types

import pytest
import torch

from gpu_util import Q

pytestmark = pytest.mark.gpu


def test_a_stream_of_another_device():
    c = Q.Cache4(1, 16, 1, 64)
    k = torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda")
    slot = torch.zeros(1, dtype=torch.int32, device="cuda")
    own = torch.cuda.Stream()
    Q.cache4_append(c, k, k, slot, stream=own)
    own.synchronize()
    with pytest.raises(ValueError, match="stream"):
        Q.cache4_append(c, k, k, slot, stream=types.SimpleNamespace(cuda_stream=0, device_index=c.device + 1))
