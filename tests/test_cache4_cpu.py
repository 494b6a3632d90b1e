"""Arguments that the cache's and the page tables' entry points refuse: each
returns its status before any device work (no GPU needed)."""
import ctypes

import pytest

FAKE = 0x10000   # never dereferenced


@pytest.fixture(scope="module")
def Q():
    from paper_2006_10226_amd import qnn
    qnn.lib()
    return qnn


def _cache(Q, **kw):
    a = dict(data=FAKE, pages=10, page_size=16, heads=2, head_dim=64)
    a.update(kw)
    return Q.Cache4Desc(a["data"], a["pages"], a["page_size"], a["heads"], a["head_dim"])


def _status(Q, code):
    msg = Q.lib().qnn_last_error().decode()
    return Q.STATUS[code], msg


CACHES = [(dict(page_size=8), "QNN_ERR_SHAPE"), (dict(page_size=48), "QNN_ERR_SHAPE"),
          (dict(page_size=512), "QNN_ERR_SHAPE"), (dict(heads=0), "QNN_ERR_SHAPE"), (dict(head_dim=0), "QNN_ERR_SHAPE"),
          (dict(head_dim=100), "QNN_ERR_SHAPE"), (dict(head_dim=264), "QNN_ERR_SHAPE"), (dict(pages=0), "QNN_ERR_SHAPE"),
          (dict(pages=2**27), "QNN_ERR_SHAPE"), (dict(data=None), "QNN_ERR_NULL"),
          (dict(data=FAKE + 8), "QNN_ERR_UNSUPPORTED")]


def test_page_bytes(Q):
    f = Q.lib().qnn_cache4_page_bytes
    assert f(16, 1, 64) == 16 * 72 and f(32, 3, 72) == 3 * 32 * 136 and f(256, 2, 256) == 2 * 256 * 264
    assert f(16, 1, 8) == 16 * 72 and f(16, 1, 136) == 16 * 264
    for bad in ((0, 1, 64), (15, 1, 64), (24, 1, 64), (-16, 1, 64), (16, 0, 64), (16, 5000, 64), (16, 1, 4), (16, 1, 260)):
        assert f(*bad) == 0


def _append(Q, cache=None, **kw):
    a = dict(k=FAKE, v=FAKE, dt=Q.FLOAT16, kq=(0.1, 0), vq=(0.1, 0), tokens=4, k_ld=128, v_ld=128, slots=FAKE)
    a.update(kw)
    kq, vq = (Q._Q(s, z, 1) for s, z in (a["kq"], a["vq"]))
    return _status(Q, Q.lib().qnn_cache4_append(None, cache or _cache(Q), a["k"], a["v"], a["dt"], kq.q, vq.q,
                                                a["tokens"], a["k_ld"], a["v_ld"], a["slots"]))


@pytest.mark.parametrize("kw,expect", CACHES)
def test_caches_refused(Q, kw, expect):
    for call in (_append, _read, _attend):
        st, msg = call(Q, _cache(Q, **kw))
        assert st == expect and msg, (call, msg)


@pytest.mark.parametrize("kw,expect", [
    (dict(k=None), "QNN_ERR_NULL"), (dict(v=None), "QNN_ERR_NULL"), (dict(slots=None), "QNN_ERR_NULL"),
    (dict(dt=2), "QNN_ERR_DTYPE"), (dict(dt=5), "QNN_ERR_DTYPE"), (dict(tokens=-1), "QNN_ERR_SHAPE"),
    (dict(k_ld=127), "QNN_ERR_SHAPE"), (dict(v_ld=0), "QNN_ERR_SHAPE"), (dict(k_ld=132), "QNN_ERR_UNSUPPORTED"),
    (dict(k=FAKE + 2), "QNN_ERR_UNSUPPORTED"), (dict(v=FAKE + 4, dt=1), "QNN_ERR_UNSUPPORTED"),
    (dict(dt=1, kq=(0.0, 0)), "QNN_ERR_QPARAM"), (dict(dt=0, vq=(0.1, -1)), "QNN_ERR_QPARAM"),
])
def test_append_refused(Q, kw, expect):
    st, msg = _append(Q, **kw)
    assert st == expect and msg


def _read(Q, cache=None, **kw):
    a = dict(slots=FAKE, tokens=4, k=FAKE, v=FAKE, dt=Q.FLOAT16, k_ld=128, v_ld=128)
    a.update(kw)
    return _status(Q, Q.lib().qnn_cache4_read(None, cache or _cache(Q), a["slots"], a["tokens"], a["k"], a["v"], a["dt"],
                                              a["k_ld"], a["v_ld"]))


@pytest.mark.parametrize("kw,expect", [
    (dict(slots=None), "QNN_ERR_NULL"), (dict(dt=1), "QNN_ERR_DTYPE"), (dict(tokens=-3), "QNN_ERR_SHAPE"),
    (dict(k_ld=64), "QNN_ERR_SHAPE"), (dict(v=FAKE + 8), "QNN_ERR_UNSUPPORTED"),
])
def test_read_refused(Q, kw, expect):
    st, msg = _read(Q, **kw)
    assert st == expect and msg


def _attend(Q, cache=None, **kw):
    a = dict(q=FAKE, qt=Q.FLOAT16, qq=(0.1, 0), table=FAKE, ctx=FAKE, cu=FAKE, tokens=4, q_heads=4, requests=2, width=8,
             q_ld=256, o_ld=256, table_ld=8, max_q=3, max_ctx=0, causal=1, window=0, scale=0.1, o=FAKE, ot=Q.FLOAT16,
             oq=(0.1, 0), ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    p = Q.AttentionParams(a["tokens"], a["q_heads"], a["requests"], a["width"], a["q_ld"], a["o_ld"], a["table_ld"],
                          a["max_q"], a["max_ctx"], a["causal"], a["window"], a["scale"])
    qq, oq = (Q._Q(s, z, 1) for s, z in (a["qq"], a["oq"]))
    return _status(Q, Q.lib().qnn_attention4(None, a["q"], a["qt"], qq.q, cache or _cache(Q), a["table"], a["ctx"],
                                             a["cu"], p, a["o"], a["ot"], oq.q, a["ws"], a["ws_bytes"]))


@pytest.mark.parametrize("kw,expect", [
    (dict(q=None), "QNN_ERR_NULL"), (dict(o=None), "QNN_ERR_NULL"), (dict(table=None), "QNN_ERR_NULL"),
    (dict(ctx=None), "QNN_ERR_NULL"), (dict(qt=2), "QNN_ERR_DTYPE"), (dict(ot=9), "QNN_ERR_DTYPE"),
    (dict(tokens=-1), "QNN_ERR_SHAPE"), (dict(requests=-1), "QNN_ERR_SHAPE"), (dict(q_heads=3), "QNN_ERR_SHAPE"),
    (dict(q_heads=0), "QNN_ERR_SHAPE"), (dict(max_q=0), "QNN_ERR_SHAPE"), (dict(max_ctx=-1), "QNN_ERR_SHAPE"),
    (dict(window=-1), "QNN_ERR_SHAPE"), (dict(width=0), "QNN_ERR_SHAPE"), (dict(table_ld=7), "QNN_ERR_SHAPE"),
    (dict(width=2**27, table_ld=2**27), "QNN_ERR_SHAPE"), (dict(q_ld=255), "QNN_ERR_SHAPE"),
    (dict(o_ld=128), "QNN_ERR_SHAPE"), (dict(cu=None), "QNN_ERR_SHAPE"), (dict(scale=float("nan")), "QNN_ERR_QPARAM"),
    (dict(scale=float("inf")), "QNN_ERR_QPARAM"), (dict(qt=1, qq=(1e30, 0), scale=1e10), "QNN_ERR_QPARAM"),
    (dict(tokens=2**30), "QNN_ERR_UNSUPPORTED"), (dict(width=2**26 + 1, table_ld=2**27), "QNN_ERR_SHAPE"), (dict(qt=1, qq=(-1.0, 0)), "QNN_ERR_QPARAM"),
    (dict(ot=0, oq=(0.1, 256)), "QNN_ERR_QPARAM"), (dict(q=FAKE + 8), "QNN_ERR_UNSUPPORTED"),
    (dict(o=FAKE + 4, ot=1), "QNN_ERR_UNSUPPORTED"), (dict(q_ld=260), "QNN_ERR_UNSUPPORTED"),
    (dict(o_ld=257), "QNN_ERR_UNSUPPORTED"), (dict(max_q=2**30), "QNN_ERR_UNSUPPORTED"),
])
def test_attention_refused(Q, kw, expect):
    st, msg = _attend(Q, **kw)
    assert st == expect and msg


def test_nothing_to_do_is_ok(Q):
    assert _append(Q, tokens=0, k=None, v=None, slots=None)[0] == "QNN_OK"
    assert _read(Q, tokens=0, slots=None)[0] == "QNN_OK"
    assert _read(Q, k=None, v=None)[0] == "QNN_OK"
    assert _attend(Q, tokens=0, q=None, o=None)[0] == "QNN_OK"
    assert _attend(Q, tokens=0, requests=0, table=None, ctx=None, cu=None)[0] == "QNN_OK"


def _resize(Q, **kw):
    a = dict(requests=2, P=16, lens=FAKE, new=FAKE, table=FAKE, width=4, ld=4, free=FAKE, cap=10, count=FAKE, cu=FAKE,
             slots=FAKE, pos=FAKE, tokens=5, status=FAKE, ws=FAKE)
    a.update(kw)
    return _status(Q, Q.lib().qnn_pages_resize(None, a["requests"], a["P"], a["lens"], a["new"], a["table"], a["width"],
                                               a["ld"], a["free"], a["cap"], a["count"], a["cu"], a["slots"], a["pos"],
                                               a["tokens"], a["status"], a["ws"]))


@pytest.mark.parametrize("kw,expect", [
    (dict(requests=-1), "QNN_ERR_SHAPE"), (dict(tokens=-1), "QNN_ERR_SHAPE"), (dict(cap=-1), "QNN_ERR_SHAPE"),
    (dict(P=0), "QNN_ERR_SHAPE"), (dict(P=24), "QNN_ERR_SHAPE"), (dict(P=8192), "QNN_ERR_SHAPE"),
    (dict(width=0), "QNN_ERR_SHAPE"), (dict(ld=3), "QNN_ERR_SHAPE"), (dict(width=2**27, ld=2**27), "QNN_ERR_UNSUPPORTED"),
    (dict(lens=None), "QNN_ERR_NULL"), (dict(new=None), "QNN_ERR_NULL"), (dict(table=None), "QNN_ERR_NULL"),
    (dict(free=None), "QNN_ERR_NULL"), (dict(count=None), "QNN_ERR_NULL"), (dict(cu=None), "QNN_ERR_NULL"),
    (dict(slots=None), "QNN_ERR_NULL"), (dict(status=None), "QNN_ERR_NULL"), (dict(ws=None), "QNN_ERR_NULL"),
    (dict(ws=FAKE + 4), "QNN_ERR_UNSUPPORTED"),
])
def test_resize_refused(Q, kw, expect):
    st, msg = _resize(Q, **kw)
    assert st == expect and msg


def test_sizes_of_workspaces(Q):
    f = Q.lib().qnn_pages_workspace_size
    assert f(-1) == 0 and f(0) > 0 and f(1000) >= 3 * 4 * 1001
    assert isinstance(ctypes.c_size_t(f(5)).value, int)


def test_the_binding_refuses_host_tensors(Q):
    import torch
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        Q.Cache4(1, 16, 1, 64, data=torch.zeros((1, 16 * 72), dtype=torch.uint8))
    with pytest.raises(ValueError):
        Q.Cache4(1, 20, 1, 64)
    with pytest.raises((ValueError, RuntimeError)):
        Q.pages_resize(i, i, i.view(1, 1), i, i, 16, 0)
