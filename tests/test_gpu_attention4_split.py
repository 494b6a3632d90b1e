"""Attention over long caches that is split over workgroups and joined, against
float64 as in test_gpu_attention4.py: several queries and one, one and two row
blocks, every padded head dimension, 16-bit and 8-bit outputs, windows, hints of
the length that are wrong, streams, graphs. Every case asserts that it is split
(a workspace is asked for)."""
import numpy as np
import pytest
import torch

from gpu_util import Q
from test_gpu_attention4 import Case

pytestmark = pytest.mark.gpu


def _split(c, a):
    T, Hq, _ = c.q.shape
    size = Q.attention4_workspace_size(c.c, T, Hq, len(c.ctx), c.W, c.max_q, a["max_ctx"], window=c.window)
    assert size > 0
    return size


LONG, QUERIES = [4000, 1700, 5], [40, 3, 5]
CASES = [
    # two row blocks, several tiles: groups that do and don't divide a tile
    dict(D=128, P=16, Hkv=1, G=1, ctx=LONG, nq=QUERIES),
    dict(D=64, P=64, Hkv=1, G=4, ctx=LONG, nq=QUERIES, qt="bf16"),
    dict(D=128, P=32, Hkv=2, G=6, ctx=LONG, nq=QUERIES),
    dict(D=256, P=128, Hkv=1, G=4, ctx=LONG, nq=QUERIES),
    dict(D=80, P=16, Hkv=3, G=5, ctx=LONG, nq=QUERIES, qt="i8"),
    # one row block of several queries
    dict(D=128, P=16, Hkv=2, G=4, ctx=[3000, 0, 1800, 2], nq=[4, 2, 1, 4]),
    dict(D=256, P=16, Hkv=1, G=1, ctx=[2000, 1999], nq=[16, 7], qt="bf16"),
    # single tokens
    dict(D=256, P=32, Hkv=2, G=3, ctx=[2600, 0, 77]),
    dict(D=64, P=16, Hkv=1, G=20, ctx=[5000, 1], qt="u8", ot="bf16"),
    # 8-bit outputs through the join
    dict(D=64, P=16, Hkv=2, G=1, ctx=[2500, 31], qt="i8"),
    dict(D=128, P=64, Hkv=1, G=4, ctx=LONG, nq=QUERIES, qt="u8"),
    dict(D=256, P=16, Hkv=1, G=2, ctx=[2000, 900], nq=[9, 1], qt="i8", ot="u8"),
    dict(D=72, P=16, Hkv=1, G=7, ctx=[1700], nq=[5], ot="i8"),
    # windows: the parts start where the first row's does
    dict(D=128, P=16, Hkv=1, G=4, ctx=LONG, nq=QUERIES, window=2000),
    dict(D=64, P=32, Hkv=2, G=2, ctx=[4000, 2100], window=1999),
    dict(D=64, P=16, Hkv=1, G=4, ctx=[6000, 30], nq=[70, 30], window=1600, qt="i8"),
    # no causal mask; with a window
    dict(D=128, P=16, Hkv=1, G=4, ctx=LONG, nq=QUERIES, causal=False),
    dict(D=64, P=16, Hkv=1, G=2, ctx=[3000, 40], nq=[20, 40], causal=False, window=1700),
    # more queries than tokens beside a long cache, a table shorter than the requests, pages of none
    dict(D=128, P=16, Hkv=1, G=2, ctx=[2500, 3], nq=[2, 30]),
    dict(D=128, P=16, Hkv=1, G=4, ctx=[4000, 60], nq=[20, 1], width=130),
    dict(D=64, P=64, Hkv=1, G=4, ctx=[3000], nq=[9], poison=[(0, 0, -1), (0, 20, 10**6), (0, 46, -7)]),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_split(i):
    c = Case(seed=100 + i, **CASES[i])
    a = c.device()
    ws = torch.full((_split(c, a),), 255, dtype=torch.uint8, device="cuda")
    y = Q.attention4(**a, workspace=ws)
    assert (ws != 255).any()
    c.check(y, f"split {i}")
    assert torch.equal(Q.attention4(**a), y)   # no sum depends on an order of execution


@pytest.mark.parametrize("nq", [[1, 1, 1], [33, 2, 5]])
@pytest.mark.parametrize("hint", [1600, 2500, 10**6])
def test_hints_of_the_length(nq, hint):
    c = Case(128, 16, 1, 4, [4000, 2000, 5], nq=nq, seed=7)
    a = c.device()
    a["max_ctx"] = hint
    _split(c, a)
    c.check(Q.attention4(**a), f"hint {hint}")


def test_queries_past_max_q_are_left():
    c = Case(128, 16, 1, 4, [3000, 1800], nq=[40, 9], seed=3)
    a = c.device()
    c.max_q = a["max_q"] = 11
    _split(c, a)
    out = torch.full(tuple(c.q.shape), 7.0, dtype=torch.float16, device="cuda")
    y = Q.attention4(**a, out=out)
    assert (y[11:40] == 7).all()
    ref, tol, _ = c.expect()
    keep = np.r_[0:11, 40:49]
    bound = tol[keep] + np.abs(ref[keep]) * 2.0**-11 * 1.01 + 2.0**-25
    assert (np.abs(y.cpu().double().numpy() - ref)[keep] <= bound).all()


def test_rows_of_no_request_and_strides():
    c = Case(64, 16, 2, 3, [2500, 1600], nq=[7, 20], extra_rows=3, seed=9)
    a = c.device()
    _split(c, a)
    T, Hq, D = c.q.shape
    out = torch.full((T, Hq * D + 24), 5.0, dtype=torch.float16, device="cuda")
    c.check(Q.attention4(**a, out=out[:, :Hq * D].unflatten(1, (Hq, D))), "strided")
    assert (out[:, Hq * D:] == 5).all() and (out[27:] == 5).all()


def test_streams_and_two_calls_at_once():
    c, d = (Case(128, 16, 2, 4, [6000, 33, 1700], nq=nq, seed=s) for s, nq in ((1, None), (2, [5, 1, 40])))
    a, b = c.device(), d.device()
    y, z = Q.attention4(**a), Q.attention4(**b)
    size = [_split(c, a), _split(d, b)]
    ws = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in size]
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        got = [Q.attention4(**a, workspace=ws[0], stream=s), Q.attention4(**b, workspace=ws[1], stream=t),
               Q.attention4(**a, stream=t), Q.attention4(**b, stream=s)]
        s.synchronize(), t.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, (y, z, y, z)))


@pytest.mark.parametrize("nq", [None, [3, 20, 1]])
def test_captured_and_replayed(nq):
    """Lengths, tables and queries that change between replays, one workspace for
    two graphs that don't overlap."""
    c = Case(128, 16, 1, 4, [4000, 1700, 900], nq=nq, seed=11)
    a = c.device()
    ws = torch.empty(_split(c, a), dtype=torch.uint8, device="cuda")
    y = Q.attention4(**a)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    outs = []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(Q.attention4(**a, workspace=ws))
    keep = a["q"].clone(), a["ctx"].clone()
    for k in range(4):
        if k % 2:
            a["q"].mul_(0.5)
            a["ctx"].sub_(torch.tensor([777, 40, 0], dtype=torch.int32, device="cuda"))
        want = Q.attention4(**a)
        for g, out in zip(graphs, outs):
            out.fill_(float("nan"))
            ws.fill_(255)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        a["q"].copy_(keep[0])
        a["ctx"].copy_(keep[1])
    assert torch.equal(Q.attention4(**a), y)


def test_a_cache_beyond_32_bits():
    """Slots whose bytes lie past 2^32, appended, read and attended to as others."""
    P, H, D, T = 256, 8, 128, 2000
    pages = 2**32 // (P * H * (D + 8)) + 20
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v, q = (torch.randn(T, H, D, generator=g, device="cuda").half() for _ in range(3))
    far, near = Q.Cache4(pages, P, H, D), Q.Cache4(8, P, H, D)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    y = []
    for c, first in ((far, pages - 8), (near, 0)):
        table = ints([first + j for j in (3, 0, 7, 1, 5, 2, 4, 6)])
        slots = (table.long()[torch.arange(T, device="cuda") // P] * P + torch.arange(T, device="cuda") % P).int()
        Q.cache4_append(c, k, v, slots)
        y.append((Q.attention4(q[:3].contiguous(), c, table.view(1, 8), ints([T]), ints([0, 3]), 3), *Q.cache4_read(c, slots)))
    assert all(torch.equal(a, b) for a, b in zip(*y))
