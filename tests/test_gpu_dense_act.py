"""Activations by table in the epilogue of matrix products
(qnn_plan_set_activation), with and without a residual add behind them, and the
lookup of its own (qnn_lookup): every byte against the oracle's product, the
table and the oracle's add; every kernel configuration, types, odd sizes, output
slices, and the plans that refuse it."""
import numpy as np
import pytest
import torch

import workloads as W
from oracle import oracle as O
from gpu_util import Q, assert_equal, dev, env, log, make_plan, run_oracle

pytestmark = pytest.mark.gpu


def _bytes(a):
    return a.view(np.uint8)


def _expect(c, table, yt):
    mid = table[_bytes(run_oracle(c))]
    return mid.view(np.int8) if yt == "i8" else mid


def _table(seed):
    return np.random.default_rng(seed).integers(0, 256, 256).astype(np.uint8)   # any function


# 1x1 convs and dense layers: channels that end inside a K-step or a chunk, one
# pixel to several tiles, ragged channels
def _cases(short):
    shapes = [(1, 64, 64), (17, 40, 72), (130, 64 * short if short else 576, 200), (300, 36, 130)]
    for i, (M, K, N) in enumerate(shapes):
        c = W.dense_case(W.DenseLayer(f"d{M}x{K}x{N}", M, K, N), seed=60 + i, yt="i8" if i % 2 else "u8",
                         zp_y=-3 if i % 2 else 120)
        if i == 3:
            c.zp_w = np.random.default_rng(5).integers(-20, 20, N).astype(np.int32)
        yield c


def _run(c, table, yt, residual=None, **kw):
    """The plan's bytes, its description; residual: (array, scale, zp, o_scale, o_zp, o_dtype)."""
    p, keep = make_plan(c, **kw)
    d = p.describe()
    p.set_activation(table, 0.05, 3, yt)
    r = None
    if residual is not None:
        r, *q = residual
        p.set_residual("u8" if r.dtype == np.uint8 else "i8", *q)
        r = dev(r)
    y = p.run(dev(c.x), residual=r)
    torch.cuda.synchronize()
    d = p.describe()
    p.close()
    return y.cpu().numpy(), d


SHORT = {10: 1, 11: 1, 12: 1, 13: 2, 14: 2, 15: 2, 16: 4, 17: 4, 18: 4, 21: 1, 22: 2}


@pytest.mark.parametrize("fam,tile", [("QNN_FLOW", t) for t in range(23)] + [("QNN_SMALL", t) for t in range(6)])
def test_every_configuration(fam, tile):
    ran = 0
    for i, c in enumerate(_cases(SHORT.get(tile, 0) if fam == "QNN_FLOW" else 0)):
        yt = ("u8", "i8")[(i + tile) % 2]
        table = _table(i)
        with env(**{fam: tile}):
            p, keep = make_plan(c)
            forced = "cands=1 " in p.describe() + " "
            p.close()
            if not forced:
                continue   # a short form with fewer stages, or a tile beyond its shapes
            ran += 1
            y, d = _run(c, table, yt)
        assert d.startswith("conv_dma_flow" if fam == "QNN_FLOW" else "conv_dma_small") and d.endswith(" +act"), d
        log(f"activation {fam}={tile} {c.name}: {d}")
        assert_equal(y, _expect(c, table, yt), f"{fam}={tile} {c.name}: {d}")
        # the same with a residual add behind it
        M, N = y.shape
        mid = _expect(c, table, yt)
        rng = np.random.default_rng(i)
        r = rng.integers(0, 256, (M, N)).astype(np.uint8)
        y_ldc = -(-N // 16) * 16
        with env(**{fam: tile}):
            y, d = _run(c, table, yt, (r, 0.0417, 100, 0.06, 90, "u8"), y_ldc=y_ldc)
        assert d.endswith(("+act +add(f32)", "+act +add")), d     # terms in f32, or by tables where they have ties
        assert_equal(y[:, :N], O.add(mid, 0.05, 3, r, 0.0417, 100, 0.06, 90, "u8", None), f"{fam}={tile} {c.name} +add: {d}")
    assert ran >= 1


@pytest.mark.parametrize("kind", ["gelu", "gelu_tanh", "silu", "sigmoid", "tanh", "hard_swish"])
@pytest.mark.parametrize("xt,yt", [("u8", "i8"), ("i8", "u8"), ("i8", "i8"), ("u8", "u8")])
def test_named_activations(kind, xt, yt):
    c = W.dense_case(W.DenseLayer("named", 33, 96, 80), seed=9, yt=xt, zp_y=-3 if xt == "i8" else 131)
    p, keep = make_plan(c)
    p.set_activation(kind, 0.02, 5, yt)
    y = p.run(dev(c.x))
    table = Q.activation_table(kind, xt, c.s_y, c.zp_y, yt, 0.02, 5)
    assert_equal(y.cpu().numpy(), _expect(c, table, yt), kind)
    assert y.dtype == (torch.int8 if yt == "i8" else torch.uint8)
    # the same in a pass of its own
    plain, keep = make_plan(c)
    z = Q.lookup(plain.run(dev(c.x)), table, yt)
    assert torch.equal(y, z)
    plain.close()
    p.close()


def test_output_slices_and_addresses():
    """Rows that are not 16-byte multiples and unaligned outputs take the
    direct stores; bytes outside the rows stay."""
    c = W.dense_case(W.DenseLayer("s", 50, 64, 61), seed=2)
    table = _table(3)
    ref = _expect(c, table, "i8")
    for fam, tile in (("QNN_FLOW", 0), ("QNN_SMALL", 1)):
        for y_ldc, shift in ((61, 0), (67, 0), (64, 1), (64, 4), (80, 0)):
            with env(**{fam: tile}):
                p, keep = make_plan(c, y_ldc=y_ldc)
            p.set_activation(table, 0.05, 3, "i8")
            buf = torch.full((50 * y_ldc + 16,), 77, dtype=torch.int8, device="cuda")
            out = buf[shift:shift + 50 * y_ldc].view(50, y_ldc)
            p.run(dev(c.x), out=out)
            torch.cuda.synchronize()
            p.close()
            assert_equal(out[:, :61].cpu().numpy(), ref, f"{fam}={tile} y_ldc {y_ldc} shift {shift}")
            assert (out[:, 61:] == 77).all() and (buf[:shift] == 77).all() and (buf[shift + 50 * y_ldc:] == 77).all()


@pytest.mark.parametrize("rounding", ["half_away", "two_stage"])
def test_roundings_and_weight_zero_points(rounding):
    c = W.conv_case(W.ConvLayer("r", 9, 9, 72, 100, 1, 1), 3, seed=4, rounding=rounding, zp_w="channel", yt="i8")
    table = _table(6)
    for forced in (dict(QNN_FLOW=3), dict(QNN_SMALL=2), dict(QNN_FLOW=9)):
        with env(**forced):
            y, d = _run(c, table, "u8")
        assert_equal(y, _expect(c, table, "u8"), f"{rounding} {d}")


def test_a_larger_product_on_its_own_choice():
    """Timed choice (the largest tile among them), then the residual's."""
    c = W.dense_case(W.DenseLayer("big", 1024, 512, 1024), seed=12)
    table = _table(8)
    mid = _expect(c, table, "i8")
    y, d = _run(c, table, "i8")
    assert_equal(y, mid, d)
    r = np.random.default_rng(0).integers(-128, 128, mid.shape).astype(np.int8)
    y, d = _run(c, table, "i8", (r, 0.031, -4, 0.06, 9, "i8"))
    assert_equal(y, O.add(mid, 0.05, 3, r, 0.031, -4, 0.06, 9, "i8", None), d)


def test_add_by_tables_behind_an_activation():
    c = W.dense_case(W.DenseLayer("t", 70, 64, 96), seed=13)
    table = _table(9)
    mid = _expect(c, table, "u8")
    r = np.random.default_rng(0).integers(-128, 128, mid.shape).astype(np.int8)
    for forced in (dict(QNN_FLOW=0), dict(QNN_FLOW=6), dict(QNN_SMALL=3)):
        with env(QNN_FLOAT_ADD=0, **forced):
            y, d = _run(c, table, "u8", (r, 0.041, -4, 0.05, 9, "i8"))
        assert d.endswith("+act +add"), d
        assert_equal(y, O.add(mid, 0.05, 3, r, 0.041, -4, 0.05, 9, "i8", None), d)


def test_captured_noalloc_and_empty():
    c = W.dense_case(W.DenseLayer("g", 40, 128, 64), seed=14)
    table = _table(1)
    ref = _expect(c, table, "i8")
    p, keep = make_plan(c)
    p.set_activation(table, 0.05, 3, "i8")
    x, y = dev(c.x), torch.zeros(40, 64, dtype=torch.int8, device="cuda")
    p.run(x, out=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(x, out=y)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert_equal(y.cpu().numpy(), ref, "replay")
    y.zero_()
    p.run_noalloc(x, y)
    torch.cuda.synchronize()
    assert_equal(y.cpu().numpy(), ref, "noalloc")
    p.close()
    w = dev(c.w)
    e = Q.dense_plan(0, 128, "u8", 0.02, 120, w, c.s_w, 0, None, c.s_y, c.zp_y, "i8")
    e.set_activation("gelu", 0.05, 3)
    assert e.run(torch.empty((0, 128), dtype=torch.uint8, device="cuda")).shape == (0, 64)
    e.close()


def test_refused():
    """Plans without the epilogue refuse it and run as before."""
    table = _table(2)
    c3 = W.conv_case(W.ConvLayer("c", 8, 8, 64, 64, 3, 3, 1, (1, 1, 1, 1)), 2, seed=1)
    c1 = W.conv_case(W.ConvLayer("p", 8, 8, 64, 64, 1, 1), 2, seed=2)
    pad = W.conv_case(W.ConvLayer("pad", 8, 8, 64, 64, 1, 1, 1, (1, 1, 1, 1)), 2, seed=2)
    dw = W.conv_case(W.ConvLayer("dw", 8, 8, 32, 32, 3, 3, 1, (1, 1, 1, 1), depthwise=True), 2, seed=3)
    for c, forced in ((c3, {}), (c1, dict(QNN_DMA=15)), (c1, dict(QNN_TILE=0)), (pad, {}), (dw, {})):
        with env(**forced):
            p, keep = make_plan(c)
        d = p.describe()
        with pytest.raises(Q.QnnError, match="UNSUPPORTED"):
            p.set_activation(table, 0.05, 3, "u8")
        assert p.describe() == d
        assert_equal(p.run(dev(c.x)).cpu().numpy(), run_oracle(c), "refused plan still runs")
        p.close()
    c32 = W.dense_case(W.DenseLayer("i", 8, 64, 64), seed=4, yt="i32")
    p, keep = make_plan(c32)
    with pytest.raises(Q.QnnError, match="UNSUPPORTED"):
        p.set_activation(table, 0.05, 3, "u8")
    with pytest.raises(ValueError):
        p.set_activation("gelu", 0.05, 3, "u8")
    p.close()
    c = W.dense_case(W.DenseLayer("o", 8, 64, 64), seed=4)
    p, keep = make_plan(c)
    p.set_residual("i8", 0.02, 1, 0.03, 2, "i8")
    with pytest.raises(Q.QnnError, match="UNSUPPORTED"):      # the activation comes first
        p.set_activation(table, 0.05, 3, "u8")
    p.close()
    p, keep = make_plan(c)
    for bad in ((0.0, 3, "u8"), (0.05, 256, "u8"), (float("nan"), 0, "i8")):
        with pytest.raises(Q.QnnError, match="QPARAM"):
            p.set_activation(table, *bad)
    with pytest.raises(Q.QnnError, match="DTYPE"):
        p.set_activation(table, 0.05, 3, "i32")
    p.set_activation(table, 0.05, 3, "u8")
    with pytest.raises(Q.QnnError, match="UNSUPPORTED"):      # twice
        p.set_activation(table, 0.05, 3, "u8")
    assert_equal(p.run(dev(c.x)).cpu().numpy(), _expect(c, table, "u8"), "after refusals")
    p.close()


@pytest.mark.parametrize("count", [0, 1, 15, 16, 17, 4096, 4097, 1000003])
@pytest.mark.parametrize("shift", [0, 3])
def test_lookup(count, shift):
    rng = np.random.default_rng(count)
    x = rng.integers(0, 256, count + shift).astype(np.uint8)
    table = _table(4)
    buf = torch.full((count + shift + 16,), 99, dtype=torch.uint8, device="cuda")
    xd = dev(x)[shift:]
    y = Q.lookup(xd, table, "u8", out=buf[shift:shift + count])
    torch.cuda.synchronize()
    assert np.array_equal(y.cpu().numpy(), table[x[shift:]])
    assert (buf[:shift] == 99).all() and (buf[shift + count:] == 99).all()
    # in place, and int8 in and out
    z = dev(x.view(np.int8))[shift:]
    Q.lookup(z, table, "i8", out=z)
    assert np.array_equal(z.cpu().numpy().view(np.uint8), table[x[shift:]])
