"""Writing and reading the 4-bit cache (qnn_cache4_append, qnn_cache4_read):
every byte of the pages against a plain model in f32, values read back, over
head dimensions, page sizes and types; slots that are skipped, strided rows,
odd values; the refusals are in test_cache4_cpu.py."""
import numpy as np
import pytest
import torch

import cache4_ref as R
from gpu_util import Q, log

pytestmark = pytest.mark.gpu

_TORCH = {"u8": torch.uint8, "i8": torch.int8, "f16": torch.float16, "bf16": torch.bfloat16}


def _rows(rng, dtype, T, H, D, ld):
    """A [T][H][D] view of rows of stride ld, its f32 values and (scale, zp)."""
    if dtype in ("u8", "i8"):
        lo = 0 if dtype == "u8" else -128
        a = torch.from_numpy(rng.integers(lo, lo + 256, (T, ld)).astype(np.int16)).to(_TORCH[dtype])
        scale, zp = np.float32(0.037), 120 if dtype == "u8" else -9
        val = (a.float().numpy() - zp) * scale
    else:
        a = torch.from_numpy(rng.normal(0.2, 1, (T, ld)).astype(np.float32)).to(_TORCH[dtype])
        scale, zp, val = 1.0, 0, a.float().numpy()
    view = a.cuda().as_strided((T, H, D), (ld, D, 1))
    return view, val[:, :H * D].reshape(T, H, D), scale, zp


def _expect(cache, slots, k, v):
    for kind, x in ((0, k), (1, v)):
        code, s, z = R.quantize(x)
        for i, slot in enumerate(slots):
            if 0 <= slot < cache.pages * cache.P:
                for h in range(cache.H):
                    cache.write(slot, h, kind, code[i, h], s[i, h], z[i, h])


def _same(got, cache):
    """Equal bytes; channels past head_dim hold anything."""
    P, D, DP = cache.P, cache.D, R.padded(cache.D)
    mask = np.zeros(P * (DP + 8), np.uint8)
    for place in (R.k_place, R.v_place):
        byte, shift = place(P, D)
        np.bitwise_or.at(mask, byte.ravel(), (15 << shift.ravel()).astype(np.uint8))
    mask[P * DP:] = 255
    a, b = got.reshape(cache.pages, cache.H, -1) & mask, cache.block() & mask
    bad = np.argwhere(a != b)
    assert bad.size == 0, (len(bad), bad[:4].tolist())


CASES = [  # dtype, T, H, D, P
    ("f16", 1, 1, 64, 16), ("bf16", 5, 3, 64, 32), ("f16", 33, 2, 128, 16), ("i8", 70, 4, 128, 64),
    ("u8", 17, 1, 256, 16), ("bf16", 130, 2, 256, 128), ("f16", 40, 3, 80, 16), ("i8", 9, 2, 8, 256),
    ("bf16", 21, 5, 136, 32), ("f16", 12, 1, 248, 16), ("u8", 50, 2, 40, 16),
]


@pytest.mark.parametrize("dtype,T,H,D,P", CASES)
def test_append_writes_the_modelled_bytes(dtype, T, H, D, P):
    rng = np.random.default_rng(T * D)
    pages = (T + P - 1) // P + 2
    cache = R.Cache(pages, P, H, D, fill=0xff)
    ld = H * D + 8 * (T % 3)
    k, kv, ks, kz = _rows(rng, dtype, T, H, D, ld)
    v, vv, vs, vz = _rows(rng, dtype, T, H, D, ld + 8)
    slots = rng.permutation(pages * P)[:T]
    slots[::5] = rng.choice([-1, -7, pages * P, 2**31 - 1], slots[::5].size)   # skipped
    c = Q.Cache4(pages, P, H, D, data=torch.from_numpy(cache.data).cuda())
    st = torch.from_numpy(slots.astype(np.int32)).cuda()
    Q.cache4_append(c, k, v, st, ks, kz, vs, vz)
    _expect(cache, slots, kv, vv)
    torch.cuda.synchronize()
    log(f"append {dtype} T={T} H={H} D={D} P={P}")
    _same(c.data.cpu().numpy(), cache)
    # read back: every slot's value rounded once, skipped ones zero
    for name in ("f16", "bf16"):
        rk, rv = Q.cache4_read(c, st, name)
        ok = (slots >= 0) & (slots < pages * P)
        for got, kind in ((rk, 0), (rv, 1)):
            for h in range(H):
                want = np.zeros((T, D))
                want[ok] = cache.read(slots[ok], h, kind)[0]
                want = torch.from_numpy(want.astype(np.float32)).to(_TORCH[name])
                assert torch.equal(got[:, h].cpu(), want), (name, kind, h)


def test_append_odd_values():
    """Zeros, constants, one-sided vectors, NaN, infinities, the largest and
    smallest values, and ties."""
    D, P = 64, 16
    rng = np.random.default_rng(1)
    x = np.zeros((14, 1, D), np.float32)
    x[1] = 3.0
    x[2] = -2.5
    x[3, 0, 5] = np.nan
    x[4] = rng.normal(size=D)
    x[4, 0, 7] = np.inf
    x[5] = rng.normal(size=D)
    x[5, 0, :2] = (-np.inf, np.nan)
    x[6, 0, ::2], x[6, 0, 1::2] = 3e38, -3e38
    x[7] = 1e-40
    x[8] = rng.normal(size=D) * 1e-39
    x[9] = np.arange(D) % 16 / 2          # steps of a half: ties
    x[10] = (np.arange(D) % 31 - 15) / 4
    x[11] = np.nan
    x[12] = rng.normal(size=D) * 1e30
    x[13] = np.abs(rng.normal(size=D)) + 5
    k = torch.from_numpy(x).to(torch.bfloat16)
    cache = R.Cache(2, P, 1, D, fill=0)
    slots = np.arange(14)
    c = Q.Cache4(2, P, 1, D, data=torch.from_numpy(cache.data).cuda())
    Q.cache4_append(c, k.cuda(), k.flip(0).contiguous().cuda(), torch.arange(14, dtype=torch.int32, device="cuda"))
    val = k.float().numpy()
    _expect(cache, slots, val, val[::-1])
    torch.cuda.synchronize()
    _same(c.data.cpu().numpy(), cache)
    rk, _ = Q.cache4_read(c, torch.arange(14, dtype=torch.int32, device="cuda"), "bf16")
    assert torch.isfinite(rk).all()
    # within a step of the input (codes are clamped at neither end by more than rounding)
    want = np.clip(np.nan_to_num(val, nan=0.0, posinf=2.0**126, neginf=-2.0**126), -2.0**126, 2.0**126)
    step = np.maximum(want.max(-1), 0) - np.minimum(want.min(-1), 0)
    # half a step from each of the value's and the zero point's rounding, then bf16's own
    off = np.abs(rk.float().cpu().numpy() - want)
    assert (off <= (step / 15 * 1.001 + np.abs(want) * 2.0**-8)[..., :] if step.ndim == want.ndim else
            off <= step[..., None] / 15 * 1.001 + np.abs(want) * 2.0**-8 + step[..., None] * 2.0**-8).all()


def test_append_on_another_stream_and_in_a_graph():
    T, H, D, P = 24, 2, 128, 16
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(T, H, D, generator=g).half().cuda() for _ in range(2))
    slots = torch.arange(T, dtype=torch.int32).flip(0).contiguous().cuda()
    ref = Q.Cache4(2, P, H, D, data=torch.zeros(2, R.page_bytes(P, H, D), dtype=torch.uint8, device="cuda"))
    Q.cache4_append(ref, k, v, slots)
    rk, rv = Q.cache4_read(ref, slots, "f16")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    c = Q.Cache4(2, P, H, D, data=torch.zeros_like(ref.data))
    with torch.cuda.stream(s):
        Q.cache4_append(c, k, v, slots)
    sk, sv = Q.cache4_read(c, slots, "f16", stream=s)
    s.synchronize()
    assert torch.equal(c.data, ref.data) and torch.equal(sk, rk) and torch.equal(sv, rv)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Q.cache4_append(c, k, v, slots)
        gk, gv = Q.cache4_read(c, slots, "f16")
    for _ in range(3):
        c.data.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.data, ref.data) and torch.equal(gk, rk) and torch.equal(gv, rv)


@pytest.mark.parametrize("dtype,low,high", [("f16", -24, 15), ("bf16", -133, 126), ("i8", 0, 0), ("u8", 0, 0)])
def test_append_codes_and_records_over_all_ranges(dtype, low, high):
    """Every code and record of 20000 vectors: their ranges over the type's, a third
    of them small integers times one step, so that quotients fall on halves."""
    T, D, P = 20000, 64, 64
    rng = np.random.default_rng(T + high)
    if dtype in ("i8", "u8"):
        first = -128 if dtype == "i8" else 0
        x = np.clip(rng.integers(-9, 10, (T, 1, D)) * rng.integers(1, 15, (T, 1, 1)) + rng.integers(0, 100, (T, 1, 1)),
                    first, first + 255)
        scale, zp = np.float32(0.037), 3
        val = (x - zp).astype(np.float32) * scale
        x = torch.from_numpy(x.astype(np.int16)).to(_TORCH[dtype])
    else:
        v = rng.normal(rng.normal(size=(T, 1, 1)), 1, (T, 1, D))
        v[::3] = rng.integers(-rng.integers(1, 30, (T, 1, 1))[::3], 31, v[::3].shape) / 8
        v *= 2.0 ** rng.integers(low, high - 3, (T, 1, 1))
        x = torch.from_numpy(v).to(_TORCH[dtype])
        scale, zp, val = 1.0, 0, x.float().numpy()
    pages = -(-T // P)
    c = Q.Cache4(pages, P, 1, D, data=torch.full((pages, R.page_bytes(P, 1, D)), 255, dtype=torch.uint8, device="cuda"))
    Q.cache4_append(c, x.cuda(), x.cuda(), torch.arange(T, dtype=torch.int32, device="cuda"), scale, zp, scale, zp)
    got = c.data.cpu().numpy()
    code, s, z = R.quantize(val[:, 0])
    rec = s.view(np.uint32) | z
    for kind, place in enumerate((R.k_place, R.v_place)):
        byte, shift = place(P, D)
        have = (got[:, byte] >> shift & 15).reshape(-1, D)[:T]
        at = P * D + 4 * P * kind
        have_rec = got[:, at:at + 4 * P].copy().view(np.uint32).reshape(-1)[:T]
        assert np.array_equal(have_rec, rec), (kind, np.flatnonzero(have_rec != rec)[:4])
        bad = np.argwhere(have != code)
        assert bad.size == 0, (kind, len(bad), bad[:4].tolist())
