"""Attention over the 4-bit cache where its numbers are far apart: a token that
outweighs a long tail, scores of any size, queries of any size. Keys and values
are written by qnn_cache4_append and known exactly, so that the softmax is too."""
import math

import numpy as np
import pytest
import torch

import cache4_ref as R
from gpu_util import Q

pytestmark = pytest.mark.gpu

_HALF_STEP = {"f16": 2.0**-11, "bf16": 2.0**-8}


def _cache(k, v, P=256):
    """A cache of one head from f32 K and V [tokens][D] that bf16 holds, the values
    as stored in float64, and its table."""
    T, D = k.shape
    pages = -(-T // P)
    c = Q.Cache4(pages, P, 1, D)
    dev = [torch.from_numpy(x).to(torch.bfloat16).cuda().unsqueeze(1).contiguous() for x in (k, v)]
    assert all(np.array_equal(d[:, 0].float().cpu().numpy(), x) for d, x in zip(dev, (k, v)))
    Q.cache4_append(c, *dev, torch.arange(T, dtype=torch.int32, device="cuda"))
    stored = []
    for x in (k, v):
        code, s, z = R.quantize(x)
        stored.append((code - z.astype(np.float64)[:, None]) * s.astype(np.float64)[:, None])
    return c, stored, torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)


def _attend(c, table, T, q, **kw):
    """q [queries][D] of one request of T tokens, all of which each of them sees."""
    n = q.shape[0]
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    y = Q.attention4(q.cuda().unsqueeze(1).contiguous(), c, table, ints(T), ints(0, n), max_q=n, causal=False, **kw)
    return y[:, 0].cpu().double().numpy()


@pytest.mark.parametrize("ot", ["f16", "i8"])
@pytest.mark.parametrize("tail", [-25.5, -24.2, -20.0])
def test_a_token_before_a_long_flat_tail(ot, tail):
    """One token outweighs each of 65535 others by 2^25 and more, but not their
    sum; the output is the tail's alone in all channels but the last."""
    T, D = 65536, 64
    k, v = np.zeros((T, D), np.float32), np.ones((T, D), np.float32)
    k[0, 0], v[0, :-1] = 1.0, 0.0
    c, (ks, vs), table = _cache(k, v)
    q = torch.zeros(1, D, dtype=torch.float16)
    q[0, 0] = -tail * math.log(2) / 0.125
    x = ks @ q[0].double().numpy() * 0.125
    p = np.exp(x - x.max())
    want = p @ vs / p.sum()
    # max_ctx: the tokens in one part, every fourth 32 of them a wave's
    o_scale = float(np.float32(want[0] / 100))
    y = _attend(c, table, T, q, max_ctx=1, scale=0.125, y_dtype=ot, y_scale=o_scale)
    # a wave's weights are f16 or its subnormals, half a step of which is 2^-25 beside
    # a largest of at least 2^7; every term's score, exponential and f32 sum over 512
    # steps: x 2^-23, 2^-20, 512 x 2^-24, of which 2^-14 is more
    tol = T / 4 * 2.0**-32 * vs.max() + want * (2.0**-11 + 2.0**-14)
    if ot == "i8":
        y, tol, want = y * o_scale, tol + o_scale * 0.51, np.minimum(want, 127 * o_scale)
    else:
        tol = tol + want * _HALF_STEP[ot]
    assert (np.abs(y[0] - want) <= tol).all(), (y[0, :3], want[:3], tol[:3])


def _means(v, ot):
    want = v.mean(0)
    # equal weights; f16 values of them, f32 sums of a few dozen
    return want, np.abs(v).max(0) * 2.0**-18 + np.abs(want) * (2.0**-11 + _HALF_STEP[ot])


@pytest.mark.parametrize("power", [10, 20, 24, 30, 60])
def test_scores_of_any_size(power):
    """Two tokens share the highest score, of up to 2^95; all others are far behind."""
    T, D = 200, 64
    rng = np.random.default_rng(power)
    k = np.zeros((T, D), np.float32)
    k[:, 0] = rng.integers(1, 5, T) * 2.0**power
    k[[31, 150], 0] = 8 * 2.0**power
    v = rng.integers(-8, 9, (T, D)).astype(np.float32)
    c, (_, vs), table = _cache(k, v)
    q = torch.zeros(64, D, dtype=torch.bfloat16)
    q[:, 0] = 2.0**min(power, 30) * (1 + torch.arange(64) / 64)
    y = _attend(c, table, T, q, scale=0.125)
    want, tol = _means(vs[[31, 150]], "bf16")
    assert (np.abs(y - want) <= tol).all(), np.abs(y - want).max()


@pytest.mark.parametrize("power", [3, 40, 59])
def test_scores_far_below_zero(power):
    """All tokens at one score, down to -2^118."""
    T, D = 64, 64
    rng = np.random.default_rng(power)
    k = np.zeros((T, D), np.float32)
    k[:, 0] = 2.0**power
    v = rng.integers(-8, 9, (T, D)).astype(np.float32)
    c, (_, vs), table = _cache(k, v)
    q = torch.zeros(3, D, dtype=torch.bfloat16)
    q[:, 0] = -(2.0**power) * torch.tensor([1.0, 1.25, 1.5])
    y = _attend(c, table, T, q, scale=0.125)
    want, tol = _means(vs, "bf16")
    assert (np.abs(y - want) <= tol).all(), np.abs(y - want).max()


@pytest.mark.parametrize("size", [1e-38, 1e30, 1e36, 3e38])
def test_queries_of_any_size_on_keys_of_zero(size):
    T, D = 64, 64
    rng = np.random.default_rng(7)
    v = rng.integers(-8, 9, (T, D)).astype(np.float32)
    c, (_, vs), table = _cache(np.zeros((T, D), np.float32), v)
    q = (torch.from_numpy(rng.uniform(-1, 1, (3, D))) * size).to(torch.bfloat16)
    q[:, 0] = size
    y = _attend(c, table, T, q, scale=0.125)
    want, tol = _means(vs, "bf16")
    assert (np.abs(y - want) <= tol).all(), np.abs(y - want).max()
