"""Attention over the 4-bit cache (qnn_attention4) against float64, value by
value with a bound derived in cache4_ref.attention: head dimensions, page sizes,
groups of heads, single tokens and prompts, causal masks and windows, rows that
see nothing, bad pages, garbage in slots that no query sees, strides, types."""
import numpy as np
import pytest
import torch

import cache4_ref as R
from gpu_util import Q, log

pytestmark = pytest.mark.gpu

_TORCH = {"u8": torch.uint8, "i8": torch.int8, "f16": torch.float16, "bf16": torch.bfloat16}
_HALF_STEP = {"f16": 2.0**-11, "bf16": 2.0**-8}


class Case:
    def __init__(self, D, P, Hkv, G, ctx, nq=None, qt="f16", ot=None, causal=True, window=0, scale=None, width=None,
                 seed=0, k_scale=0.3, v_scale=0.1, extra_rows=0, gain=1.0, poison=()):
        rng = np.random.default_rng(seed + D)
        self.D, self.P, self.Hkv, self.G = D, P, Hkv, G
        self.qt, self.ot, self.causal, self.window = qt, ot or qt, causal, window
        self.ctx, nq = np.asarray(ctx), np.asarray(nq if nq is not None else [1] * len(ctx))
        self.cu = np.concatenate([[0], np.cumsum(nq)])
        self.max_q = max(1, int(nq.max()))
        self.scale = D ** -0.5 if scale is None else scale
        have = (self.ctx + P - 1) // P
        self.W = width or max(1, int(have.max()))
        pages = int(np.minimum(have, self.W).sum()) + 3
        perm = rng.permutation(pages)
        self.table = rng.integers(-5, pages + 5, (len(ctx), self.W))     # past the length: anything
        self.cache = R.Cache(pages, P, Hkv, D)
        at = 0
        for b, n in enumerate(self.ctx):
            m = min(int(have[b]), self.W)
            self.table[b, :m] = perm[at:at + m]
            at += m
            t = np.arange(min(int(n), m * P))
            self.cache.fill_random(self.table[b, t // P] * P + t % P, rng, k_scale, v_scale)
        for b, j, value in poison:
            self.table[b, j] = value
        T = int(self.cu[-1]) + extra_rows
        Hq = Hkv * G
        if qt in ("u8", "i8"):
            lo = 0 if qt == "u8" else -128
            self.q = torch.from_numpy(rng.integers(lo, lo + 256, (T, Hq, D)).astype(np.int16)).to(_TORCH[qt])
            self.q_scale, self.q_zp = float(np.float32(0.015 * gain)), 121 if qt == "u8" else 7
            self.q64 = (self.q.double().numpy() - self.q_zp) * self.q_scale
        else:
            self.q = torch.from_numpy(rng.normal(0, gain, (T, Hq, D)).astype(np.float32)).to(_TORCH[qt])
            self.q_scale, self.q_zp = 1.0, 0
            self.q64 = self.q.double().numpy()
        self.o_scale, self.o_zp = 0.011, 133 if self.ot == "u8" else -6

    def device(self):
        self.c = Q.Cache4(self.cache.pages, self.P, self.Hkv, self.D, data=torch.from_numpy(self.cache.data).cuda())
        put = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()  # noqa: E731
        return dict(q=self.q.cuda(), cache=self.c, block_table=put(self.table), ctx=put(self.ctx), cu_q=put(self.cu),
                    max_q=self.max_q, max_ctx=int(self.ctx.max()), scale=self.scale, causal=self.causal,
                    window=self.window, q_scale=self.q_scale, q_zp=self.q_zp, y_scale=self.o_scale, y_zp=self.o_zp,
                    y_dtype=self.ot)

    def expect(self):
        return R.attention(self.q64, self.cache, self.table, self.ctx, self.cu, self.scale, self.causal, self.window)

    def check(self, y, what=""):
        ref, tol, rows = self.expect()
        got = y.cpu()
        if self.ot in ("u8", "i8"):
            lo = 0 if self.ot == "u8" else -128
            s = float(np.float32(self.o_scale))
            got = (got.double().numpy() - self.o_zp) * s
            ref = np.clip(ref, (lo - self.o_zp) * s, (lo + 255 - self.o_zp) * s)
            tol = tol + s * (0.5 + 1e-5)
        else:
            got = got.double().numpy()
            tol = tol + np.abs(ref) * _HALF_STEP[self.ot] * 1.01 + 2.0**-25
        off = np.abs(got - ref)[rows]
        bad = ~(off <= tol[rows])
        log(f"attention {what} worst {np.nanmax(off / tol[rows]) if off.size else 0:.3f} of the bound")
        assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), off[bad][:4], tol[rows][bad][:4])
        return got


SINGLE = [
    # the shortest ones, a step's edges, pages that end inside a step
    Case(64, 16, 1, 1, [1]), Case(128, 16, 2, 4, [1, 2, 31, 32, 33, 0]), Case(128, 32, 1, 8, [127, 128, 129]),
    Case(256, 16, 1, 2, [70, 3]), Case(64, 64, 3, 5, [300, 17, 64], qt="bf16"), Case(128, 128, 2, 16, [500, 129]),
    Case(128, 256, 1, 32, [700]), Case(256, 64, 2, 20, [250, 1], qt="bf16"), Case(80, 16, 2, 3, [45, 260]),
    Case(8, 16, 1, 1, [40]), Case(40, 32, 2, 2, [99], qt="bf16"), Case(136, 16, 1, 4, [130, 16]),
    Case(248, 16, 1, 1, [50]),
    Case(64, 16, 2, 2, [513, 100], qt="i8"), Case(128, 16, 1, 4, [90, 400], qt="u8"),
    Case(128, 32, 2, 4, [333], qt="i8", ot="bf16"), Case(64, 16, 2, 1, [64, 65], qt="f16", ot="i8"),
    Case(256, 32, 1, 3, [200], qt="u8", ot="f16"), Case(128, 16, 1, 2, [150], qt="bf16", ot="u8"),
    Case(128, 16, 2, 4, [3000, 5, 1700, 0, 2999]), Case(64, 64, 1, 8, [4100], qt="bf16"),
]


@pytest.mark.parametrize("i", range(len(SINGLE)))
def test_single_tokens(i):
    c = SINGLE[i]
    a = c.device()
    c.check(Q.attention4(**a), f"single {i}")
    # one query each needs no cu_q
    a["cu_q"] = None
    c.check(Q.attention4(**a), f"single {i} without cu_q")


PROMPTS = [
    dict(D=128, P=16, Hkv=1, G=4, ctx=[40], nq=[40]),
    dict(D=64, P=32, Hkv=2, G=1, ctx=[100, 17, 65], nq=[33, 17, 1]),
    dict(D=128, P=64, Hkv=1, G=8, ctx=[300, 20, 90], nq=[20, 0, 90], qt="bf16"),
    dict(D=256, P=16, Hkv=1, G=2, ctx=[70, 130], nq=[70, 9]),
    dict(D=80, P=16, Hkv=2, G=3, ctx=[64, 33], nq=[31, 33], qt="i8", ot="i8"),
    dict(D=128, P=16, Hkv=1, G=4, ctx=[5, 0, 30], nq=[9, 4, 30]),            # more queries than tokens: empty rows
    dict(D=128, P=16, Hkv=1, G=4, ctx=[60, 41], nq=[50, 41], causal=False),
    dict(D=64, P=16, Hkv=1, G=4, ctx=[200, 77], nq=[60, 77], window=33),
    dict(D=128, P=32, Hkv=2, G=2, ctx=[150, 64], nq=[5, 64], window=1),
    dict(D=128, P=16, Hkv=1, G=6, ctx=[90], nq=[40], window=500, qt="u8", ot="f16"),
    dict(D=64, P=128, Hkv=1, G=16, ctx=[400], nq=[130]),
    dict(D=64, P=16, Hkv=1, G=2, ctx=[100], nq=[10], causal=False, window=40),
]


@pytest.mark.parametrize("i", range(len(PROMPTS)))
def test_prompts(i):
    c = Case(seed=i, **PROMPTS[i])
    c.check(Q.attention4(**c.device()), f"prompt {i}")


def test_window_of_single_tokens():
    c = Case(128, 16, 2, 4, [1000, 50, 31, 1, 0], window=50)
    c.check(Q.attention4(**c.device()), "window")


def test_slots_outside_the_window_may_hold_anything():
    """Pages that slid out of the window have been given up: table entries -1, or
    pages of others with NaN records."""
    c = Case(128, 16, 1, 4, [200], window=40, poison=[(0, j, (-1, 10**6, 0)[j % 3]) for j in range(9)])
    spare = [p for p in range(c.cache.pages) if p not in set(c.table[0, 9:])]
    c.table[0, 2] = spare[0]
    c.cache.data[spare[0]] = 0xff
    y = Q.attention4(**c.device())
    assert torch.isfinite(y).all()
    c.check(y, "slid")


def test_bad_pages_are_not_seen():
    for value in (-1, 10**8, -2**31, 2**31 - 1):
        c = Case(128, 16, 1, 4, [100, 64], poison=[(0, 2, value), (0, 5, value), (1, 0, value)])
        c.check(Q.attention4(**c.device()), f"page {value}")
    c = Case(64, 32, 1, 1, [64], poison=[(0, 0, -1), (0, 1, -1)])
    y = Q.attention4(**c.device())
    assert not y.any()


def test_longer_than_the_table():
    """Tokens past the table's width are not seen."""
    c = Case(64, 16, 1, 2, [100, 40], width=4)
    c.check(Q.attention4(**c.device()), "cut")


def test_max_ctx_is_a_hint():
    c = Case(128, 16, 2, 4, [2000, 700, 64])
    for hint in (0, 1, 64, 1999, 10**6):
        a = c.device()
        a["max_ctx"] = hint
        c.check(Q.attention4(**a), f"max_ctx {hint}")


def test_rows_of_no_request_stay():
    c = Case(128, 16, 1, 4, [50, 20], nq=[3, 2], extra_rows=4)
    out = torch.full((9, 4, 128), 7.0, dtype=torch.float16, device="cuda")
    y = Q.attention4(**c.device(), out=out)
    c.check(y, "behind")
    assert (out[5:] == 7).all()


def test_queries_past_max_q_are_left():
    """max_q below a request's queries: the first ones are computed, at their own
    positions, the rest stays."""
    c = Case(128, 16, 2, 4, [90, 33, 40], nq=[20, 3, 40])
    for most in (1, 3, 17):
        a = c.device()
        a["max_q"] = most
        out = torch.full(tuple(c.q.shape), 7.0, dtype=torch.float16, device="cuda")
        y = Q.attention4(**a, out=out).cpu().double().numpy()
        ref, tol, _ = c.expect()
        for b in range(3):
            lo, hi = int(c.cu[b]), int(c.cu[b + 1])
            mid = min(hi, lo + most)
            bound = tol[lo:mid] + np.abs(ref[lo:mid]) * _HALF_STEP["f16"] * 1.01 + 2.0**-25
            assert (np.abs(y[lo:mid] - ref[lo:mid]) <= bound).all(), (most, b)
            assert (y[mid:hi] == 7).all(), (most, b)


def test_a_query_that_is_not_finite():
    """Its own rows only; 8-bit outputs of it are the zero point."""
    for ot in ("f16", "i8"):
        c = Case(64, 16, 1, 4, [50, 60], ot=ot)
        good = Q.attention4(**c.device())
        c.q[0, 1, 5], c.q[0, 2, 63] = float("nan"), float("inf")
        y = Q.attention4(**c.device())
        assert torch.equal(y[0, 0], good[0, 0]) and torch.equal(y[0, 3], good[0, 3]) and torch.equal(y[1], good[1])
        if ot == "i8":
            assert (y[0, 1] == c.o_zp).all()
        else:
            assert torch.isnan(y[0, 1]).all()


def test_workspaces():
    """A workspace of the given size serves; a smaller one is refused."""
    c = Case(128, 16, 1, 4, [6000, 900])
    a = c.device()
    y = Q.attention4(**a)
    size = Q.attention4_workspace_size(c.c, 2, 4, 2, c.W, 1, a["max_ctx"])
    assert size > 0
    ws = torch.full((size + 32,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(Q.attention4(**a, workspace=ws[:size]), y)
    assert (ws[size:] == 255).all()
    with pytest.raises(Q.QnnError, match="SHAPE"):
        Q.attention4(**a, workspace=ws[:size - 16])
    with pytest.raises(Q.QnnError, match="UNSUPPORTED"):
        Q.attention4(**a, workspace=ws[4:4 + size])


def test_strided_rows_and_tables():
    c = Case(128, 16, 2, 2, [90, 33, 150], nq=[4, 1, 9])
    a = c.device()
    T, Hq, D = a["q"].shape
    wide = torch.full((T, (Hq + 4) * D), 9.0, dtype=torch.float16, device="cuda")
    wide[:, 2 * D:(Hq + 2) * D] = a["q"].reshape(T, -1)
    a["q"] = wide[:, 2 * D:(Hq + 2) * D].unflatten(1, (Hq, D))
    t = torch.full((3, c.W + 5), -9, dtype=torch.int32, device="cuda")
    t[:, :c.W] = a["block_table"]
    a["block_table"] = t[:, :c.W]
    out = torch.full((T, (Hq + 1) * D), 5.0, dtype=torch.float16, device="cuda")
    y = Q.attention4(**a, out=out[:, :Hq * D].unflatten(1, (Hq, D)))
    c.check(y, "strided")
    assert (out[:, Hq * D:] == 5).all()


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0, 1e-6])
def test_scales(scale):
    c = Case(64, 16, 1, 4, [77, 5], scale=scale)
    c.check(Q.attention4(**c.device()), f"scale {scale}")


@pytest.mark.parametrize("k_scale,v_scale,gain,qt", [(0.3, 1e-25, 1, "f16"), (0.3, 1e25, 1, "bf16"), (3.0, 0.1, 8, "f16"),
                                                     (1e-3, 50.0, 1e3, "f16"), (1e-20, 0.1, 1e19, "bf16"),
                                                     (1e8, 0.1, 1e-7, "f16")])
def test_sizes_of_values(k_scale, v_scale, gain, qt):
    """Scales far from 1 (outputs in bf16, whose range holds them), sharp softmaxes."""
    c = Case(128, 16, 1, 4, [300, 41], k_scale=k_scale, v_scale=v_scale, gain=gain, qt=qt, ot="bf16")
    c.check(Q.attention4(**c.device()), f"values {k_scale} {v_scale} {gain}")


def test_scales_of_v_that_differ():
    """Tokens whose V scale is 2^40 larger than the rest's but which hardly weigh,
    zero vectors, and the other way round."""
    c = Case(64, 16, 1, 2, [64], seed=5)
    b = c.cache.block()
    at = c.P * 64 + 4 * c.P

    def put(t, scale):
        rec = int(np.float32(scale).view(np.uint32)) & 0xffffff00 | 7
        b[c.table[0, t // 16], 0, at + 4 * (t % 16):at + 4 * (t % 16) + 4] = np.frombuffer(np.uint32(rec).tobytes(), np.uint8)

    for t, s in ((0, 2.0**30), (7, 0.0), (33, 2.0**-60), (40, 2.0**-30)):
        put(t, s)
    c.ot = "bf16"
    c.check(Q.attention4(**c.device()), "uneven V")


def test_streams_and_repeats():
    c = Case(128, 16, 2, 4, [900, 33, 400])
    a = c.device()
    y = Q.attention4(**a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        z = Q.attention4(**a)
    w = Q.attention4(**a, stream=s)
    s.synchronize()
    assert torch.equal(y, z) and torch.equal(y, w)


def test_captured_and_replayed():
    c = Case(128, 16, 2, 4, [900, 33, 400])
    a = c.device()
    y = Q.attention4(**a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = Q.attention4(**a)
    q = a["q"]
    for k in range(3):
        keep = q.clone()
        if k == 1:
            q.mul_(0.5)
        want = Q.attention4(**a)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want)
        q.copy_(keep)
    assert torch.equal(Q.attention4(**a), y)
