"""Block tables and slots (qnn_pages_resize) against a plain model, whole
numbers compared for equality: growth, shrinking, both at once, shortages and
bad lengths that change nothing, one request to thousands, captured steps."""
import numpy as np
import pytest
import torch

from gpu_util import Q, log

pytestmark = pytest.mark.gpu


class Model:
    """Request lengths, their table and the free stack."""

    def __init__(self, B, W, P, pages, rng, lens, spare=0):
        self.P, self.W = P, W
        perm = list(rng.permutation(pages))
        self.lens = np.asarray(lens, np.int64)
        self.table = rng.integers(-9, 10**9, (B, W))
        for b in range(B):
            for j in range(-(-int(self.lens[b]) // P)):
                self.table[b, j] = perm.pop()
        self.free = perm
        self.capacity = pages + spare
        self.stack = rng.integers(-9, 10**9, self.capacity)
        self.stack[:len(perm)] = perm

    def resize(self, new, tokens):
        """(cu, slots, positions, status); the model's state moves on."""
        B, P = len(self.lens), self.P
        cu, slots, pos = np.zeros(B + 1, np.int64), np.full(tokens, -1), np.zeros(tokens, np.int64)
        most, n = self.W * P, len(self.free)
        if (self.lens < 0).any() or (self.lens > most).any() or (new < 0).any() or (new > most).any():
            return cu, slots, pos, -1
        have, want = -(-self.lens // P), -(-new // P)
        if np.maximum(new - self.lens, 0).sum() > tokens:
            return cu, slots, pos, -2
        if n + np.maximum(have - want, 0).sum() > self.capacity:
            return cu, slots, pos, -3
        short = np.maximum(want - have, 0).sum() - n - np.maximum(have - want, 0).sum()
        if short > 0:
            return cu, slots, pos, short
        back = [(b, j) for b in range(B) for j in range(want[b], have[b])]
        for i, (b, j) in enumerate(back):
            self.stack[n + len(back) - 1 - i] = self.table[b, j]
            self.table[b, j] = -1
        top = n + len(back)
        for b in range(B):
            for j in range(have[b], want[b]):
                top -= 1
                self.table[b, j] = self.stack[top]
        at = 0
        for b in range(B):
            cu[b] = at
            for p in range(self.lens[b], new[b]):
                slots[at], pos[at] = self.table[b, p // P] * P + p % P, p
                at += 1
        cu[B] = at
        self.lens = new.copy()
        self.free = list(self.stack[:top])
        return cu, slots, pos, 0


class Device:
    def __init__(self, m):
        put = lambda a: torch.from_numpy(np.ascontiguousarray(a).astype(np.int32)).cuda()  # noqa: E731
        self.m, self.put = m, put
        wide = np.full((m.table.shape[0], m.W + 3), 12345)
        wide[:, :m.W] = m.table
        self.wide = put(wide)
        self.lens, self.table = put(m.lens), self.wide[:, :m.W]
        self.stack, self.count = put(m.stack), put([len(m.free)])

    def step(self, new, tokens, what):
        got = Q.pages_resize(self.lens, self.put(new), self.table, self.stack, self.count, self.m.P, tokens)
        torch.cuda.synchronize()
        self.compare([x.cpu().numpy() for x in got], self.m.resize(new, tokens), what)

    def compare(self, got, want, what):
        m = self.m
        log(f"pages {what}: status {want[3]}, {want[0][-1]} tokens")
        assert got[3] == want[3], (what, got[3], want[3])
        for name, g, w in zip(("cu", "slots", "positions"), got, want):
            assert np.array_equal(g, w), (what, name, np.argwhere(g != w)[:4].tolist())
        assert np.array_equal(self.lens.cpu().numpy(), m.lens), what
        assert np.array_equal(self.table.cpu().numpy(), m.table), what
        assert np.array_equal(self.stack.cpu().numpy(), m.stack), what
        assert int(self.count) == len(m.free), what
        assert (self.wide[:, m.W:] == 12345).all()


@pytest.mark.parametrize("B,W,P", [(1, 1, 1), (1, 40, 16), (3, 7, 16), (64, 20, 32), (65, 9, 128), (1000, 12, 16),
                                   (1024, 3, 4), (1025, 5, 2), (5000, 4, 16), (2, 3, 4096)])
def test_steps(B, W, P):
    rng = np.random.default_rng(B + W)
    most = W * P
    m = Model(B, W, P, B * W, rng, rng.integers(0, most + 1, B))
    d = Device(m)
    d.step(np.minimum(m.lens + 1, most), B + 5, "one token each")
    d.step(rng.integers(0, most + 1, B), B * most, "all at once")
    d.step(np.where(rng.random(B) < 0.5, 0, m.lens), 0, "half of them end, no new tokens")
    d.step(m.lens.copy(), 3, "nothing")
    d.step(np.full(B, most), B * most + 70, "all full")
    d.step(np.zeros(B, np.int64), 1, "all empty")


def test_giving_back_undoes_taking():
    rng = np.random.default_rng(3)
    m = Model(50, 16, 16, 800, rng, rng.integers(0, 100, 50))
    d = Device(m)
    old, stack = m.lens.copy(), m.stack.copy()
    d.step(old + rng.integers(0, 150, 50), 50 * 150, "grow")
    d.step(old, 0, "undo")
    assert np.array_equal(m.stack, stack)


def test_refused_on_the_device_changes_nothing():
    rng = np.random.default_rng(4)
    for new, tokens, free, spare, what in (
            ([200, 10, 10], 1000, 3, 5, "pages missing"), ([-1, 10, 10], 100, 30, 5, "negative"),
            ([10, 321, 10], 1000, 30, 5, "past the table"), ([60, 60, 60], 20, 30, 5, "tokens beyond the capacity"),
            ([0, 10, 10], 10, 30, -31, "stack too small")):
        m = Model(3, 20, 16, 30 + 6, rng, [20, 16, 33], spare=0)
        del m.free[free:]
        m.capacity = max(len(m.free), m.capacity + spare)
        m.stack = m.stack[:m.capacity]
        Device(m).step(np.asarray(new), tokens, what)


@pytest.mark.parametrize("lens,count", [([-5, 3], 2), ([3, 700], 2), ([1, 1], -1), ([1, 1], 100)])
def test_bad_state_changes_nothing(lens, count):
    rng = np.random.default_rng(5)
    m = Model(2, 20, 16, 8, rng, [1, 1])
    m.lens = np.asarray(lens)
    d = Device(m)
    d.count.fill_(count)
    got = Q.pages_resize(d.lens, d.put([40, 40]), d.table, d.stack, d.count, 16, 100)
    torch.cuda.synchronize()
    assert int(got[3]) == -1 and int(d.count) == count and (got[1] == -1).all() and not got[0].any()
    assert np.array_equal(d.table.cpu().numpy(), m.table) and np.array_equal(d.lens.cpu().numpy(), lens)


def test_no_requests():
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    cu, slots, pos, status = Q.pages_resize(e, e, torch.empty((0, 4), dtype=torch.int32, device="cuda"), e, count, 16, 9)
    assert cu.tolist() == [0] and slots.tolist() == [-1] * 9 and pos.tolist() == [0] * 9 and status.tolist() == [0]


def test_captured_steps():
    """A captured step, replayed: every replay adds a token to every request."""
    rng = np.random.default_rng(6)
    B, W, P = 30, 8, 16
    m = Model(B, W, P, B * W, rng, rng.integers(0, 100, B))
    d = Device(m)
    new = d.lens + 1
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = Q.pages_resize(d.lens, new, d.table, d.stack, d.count, P, B)
    for k in range(20):
        graph.replay()
        torch.cuda.synchronize()
        d.compare([x.cpu().numpy() for x in got], m.resize(m.lens + 1, B), f"replay {k}")
        new += 1


def test_on_another_stream():
    rng = np.random.default_rng(7)
    m = Model(40, 6, 16, 240, rng, rng.integers(0, 60, 40))
    d = Device(m)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    new = m.lens + 3
    arg = d.put(new)
    torch.cuda.synchronize()
    got = Q.pages_resize(d.lens, arg, d.table, d.stack, d.count, 16, 200, stream=s)
    s.synchronize()
    d.compare([x.cpu().numpy() for x in got], m.resize(new, 200), "another stream")
