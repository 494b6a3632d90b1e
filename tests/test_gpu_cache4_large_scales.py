"""qnn_cache4_append of 8-bit rows whose scale takes their values beyond +-2^126:
they count as that, as 16-bit ones do, and the records stay finite."""
import numpy as np
import pytest
import torch

import cache4_ref as R
from gpu_util import Q
from test_gpu_cache4 import _expect, _same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["i8", "u8"])
@pytest.mark.parametrize("scale", [2.0**117, 1.5 * 2.0**118, 2e36, 3e38])
def test_values_beyond_the_largest(dtype, scale):
    T, H, D, P = 12, 2, 64, 16
    rng = np.random.default_rng(5)
    zp = 9 if dtype == "i8" else 130
    lo = -128 if dtype == "i8" else 0
    x = rng.integers(lo, lo + 256, (2, T, H, D))
    x[0, 3] = zp                      # zeros
    x[1, 4] = np.maximum(x[1, 4], zp)   # one-sided
    x[0, 5] = zp + rng.integers(-3, 4, (H, D))
    scale = np.float32(scale)
    with np.errstate(over="ignore"):
        val = (x - zp).astype(np.float32) * scale
    k, v = torch.from_numpy(x.astype(np.int16)).to(torch.int8 if dtype == "i8" else torch.uint8).cuda().unbind(0)
    cache = R.Cache(2, P, H, D, fill=0)
    slots = rng.permutation(2 * P)[:T]
    c = Q.Cache4(2, P, H, D, data=torch.from_numpy(cache.data).cuda())
    Q.cache4_append(c, k, v, torch.from_numpy(slots.astype(np.int32)).cuda(), scale, zp, scale, zp)
    _expect(cache, slots, *val)
    torch.cuda.synchronize()
    _same(c.data.cpu().numpy(), cache)
    assert all(torch.isfinite(t).all() for t in Q.cache4_read(c, torch.from_numpy(slots.astype(np.int32)).cuda(), "bf16"))
