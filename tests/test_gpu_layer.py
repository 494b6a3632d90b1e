"""A quantized transformer layer as a server runs it: block tables for a batch of
prompts, then single tokens; query, key and value from one int8 dense layer, K
and V appended to the 4-bit cache from slices of its rows, attention, the output
projection with its residual, and the feed-forward pair with GELU and residual.
Every step is checked against plain models: dense layers and adds byte for byte
on the tensors that the GPU handed on, the cache byte for byte, attention within
its bound."""
import numpy as np
import pytest
import torch

import cache4_ref as R
from gpu_util import O, Q, assert_equal, log

pytestmark = pytest.mark.gpu

HID, HQ, HKV, D, P, W = 256, 4, 2, 64, 16, 6
NQKV = (HQ + 2 * HKV) * D


class Dense:
    """An int8 dense layer, its plans by number of rows."""

    def __init__(self, rng, K, N, s_y, zp_y, gelu=None, residual=None):
        self.K, self.N, self.s_y, self.zp_y, self.gelu, self.residual = K, N, s_y, zp_y, gelu, residual
        self.w = np.clip(np.rint(rng.normal(0, 30, (N, K))), -127, 127).astype(np.int8)
        self.s_w = np.exp(rng.uniform(np.log(1e-3), np.log(3e-3), N)).astype(np.float32)
        self.b = rng.integers(-3000, 3000, N).astype(np.int32)
        self.dev = [torch.from_numpy(a).cuda() for a in (self.w, self.b)]
        self.plans = {}

    def plan(self, M, s_x, zp_x):
        if M not in self.plans:
            p = Q.dense_plan(M, self.K, "i8", s_x, zp_x, self.dev[0], self.s_w, 0, self.dev[1], self.s_y, self.zp_y, "i8")
            if self.gelu:
                p.set_activation("gelu", *self.gelu)
            if self.residual:
                p.set_residual("i8", *self.residual, "i8")
            self.plans[M] = p
        return self.plans[M]

    def expect(self, x, s_x, zp_x, r=None):
        y = O.dense(x, s_x, zp_x, self.w, self.s_w, np.zeros(self.N, np.int32), self.b, self.s_y, self.zp_y, "i8")
        if self.gelu:
            y = Q.activation_table("gelu", "i8", self.s_y, self.zp_y, "i8", *self.gelu)[y.view(np.uint8)].view(np.int8)
        if self.residual:
            s_r, zp_r, s_o, zp_o = self.residual
            s_c, zp_c = self.gelu or (self.s_y, self.zp_y)
            y = O.add(y, s_c, zp_c, r, s_r, zp_r, s_o, zp_o, "i8", None)
        return y


X = (0.03, 2)          # the layer's input
QKV = (0.02, -3)
ATT = (0.012, 5)
HIDDEN = (0.05, -1)    # after the attention block
UP, ACT = (0.06, 3), (0.04, -90)
OUT = (0.07, 4)


class Layer:
    def __init__(self, B):
        rng = np.random.default_rng(8)
        self.B = B
        self.qkv = Dense(rng, HID, NQKV, *QKV)
        self.proj = Dense(rng, HQ * D, HID, 0.03, 1, residual=(*X, *HIDDEN))
        self.up = Dense(rng, HID, 4 * HID, *UP, gelu=ACT)
        self.down = Dense(rng, 4 * HID, HID, 0.05, 0, residual=(*HIDDEN, *OUT))
        pages = B * W
        self.cache = Q.Cache4(pages, P, HKV, D)
        self.cache.data.fill_(255)
        self.model = R.Cache(pages, P, HKV, D)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.lens, self.table = torch.zeros(B, **i32), torch.full((B, W), -1, **i32)
        self.free = torch.from_numpy(rng.permutation(pages).astype(np.int32)).cuda()
        self.count = torch.tensor([pages], **i32)

    def step(self, x, new, T, max_q):
        """The GPU's tensors of one step: T new tokens, requests of new[b] tokens then."""
        cu, slots, pos, status = Q.pages_resize(self.lens, new, self.table, self.free, self.count, P, T)
        qkv = self.qkv.plan(T, *X).run(x)
        heads = qkv.view(T, HQ + 2 * HKV, D)
        q, k, v = heads[:, :HQ], heads[:, HQ:HQ + HKV], heads[:, HQ + HKV:]
        Q.cache4_append(self.cache, k, v, slots, *QKV, *QKV)
        att = Q.attention4(q, self.cache, self.table, self.lens, cu, max_q, W * P, q_scale=QKV[0], q_zp=QKV[1],
                           y_scale=ATT[0], y_zp=ATT[1])
        hidden = self.proj.plan(T, *ATT).run(att.view(T, HQ * D), residual=x)
        up = self.up.plan(T, *HIDDEN).run(hidden)
        out = self.down.plan(T, *ACT).run(up, residual=hidden)
        return dict(cu=cu, slots=slots, status=status, qkv=qkv, att=att, hidden=hidden, up=up, out=out)

    def check(self, x, t, what):
        t = {k: v.cpu().numpy() for k, v in t.items()}
        x, T = x.cpu().numpy(), x.shape[0]
        assert t["status"] == 0 and t["cu"][-1] == T and len(set(t["slots"])) == T
        assert_equal(t["qkv"], self.qkv.expect(x, *X), what + " qkv")
        h = ((t["qkv"].astype(np.float32) - QKV[1]) * np.float32(QKV[0])).reshape(T, HQ + 2 * HKV, D)
        for kind, at in ((0, HQ), (1, HQ + HKV)):
            code, s, z = R.quantize(h[:, at:at + HKV])
            for i, slot in enumerate(t["slots"]):
                for j in range(HKV):
                    self.model.write(slot, j, kind, code[i, j], s[i, j], z[i, j])
        assert np.array_equal(self.cache.data.cpu().numpy(), self.model.data), what + " cache"
        q = (t["qkv"].astype(np.float64) - QKV[1]).reshape(T, -1, D)[:, :HQ] * float(np.float32(QKV[0]))
        ref, tol, _ = R.attention(q, self.model, self.table.cpu().numpy(), self.lens.cpu().numpy(), t["cu"], D ** -0.5)
        s = float(np.float32(ATT[0]))
        ref = np.clip(ref, (-128 - ATT[1]) * s, (127 - ATT[1]) * s)
        off = np.abs((t["att"].astype(np.float64) - ATT[1]) * s - ref)
        assert (off <= tol + s * (0.5 + 1e-5)).all(), (what, off.max(), s)
        assert_equal(t["hidden"], self.proj.expect(t["att"].reshape(T, -1), *ATT, r=x), what + " projection")
        assert_equal(t["up"], self.up.expect(t["hidden"], *HIDDEN), what + " up")
        assert_equal(t["out"], self.down.expect(t["up"], *ACT, r=t["hidden"]), what + " down")
        log(f"layer {what}: {T} tokens")


def _x(seed, T):
    return torch.from_numpy(np.random.default_rng(seed).integers(-128, 128, (T, HID)).astype(np.int8)).cuda()


def test_prompts_then_single_tokens():
    B = 5
    layer = Layer(B)
    lens = np.array([33, 1, 70, 16, 5])
    x = _x(1, int(lens.sum()))
    new = torch.from_numpy(lens.astype(np.int32)).cuda()
    t = layer.step(x, new, x.shape[0], int(lens.max()))
    torch.cuda.synchronize()
    layer.check(x, t, "prompts")
    for k in range(2):                      # single tokens, eager
        x = _x(2 + k, B)
        t = layer.step(x, layer.lens + 1, B, 1)
        torch.cuda.synchronize()
        layer.check(x, t, f"token {k}")
    # and captured: every replay is a token more
    x, new = _x(9, B), layer.lens + 1
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t = layer.step(x, new, B, 1)
    for k in range(14):                     # across the end of a page
        x.copy_(_x(20 + k, B))
        graph.replay()
        torch.cuda.synchronize()
        layer.check(x, t, f"replay {k}")
        new += 1
    # a request ends, its pages go to another
    x = _x(40, 20)
    new = layer.lens.clone()
    new[2], new[1] = 0, new[1] + 20
    t = layer.step(x, new, 20, 20)
    torch.cuda.synchronize()
    layer.check(x, t, "batch changes")
