"""Plain model of the 4-bit cache and its operators (include/qnn.h), for their
tests: numpy, attention in float64."""
import numpy as np


def padded(D):
    return 64 if D <= 64 else 128 if D <= 128 else 256


def page_bytes(P, H, D):
    return H * P * (padded(D) + 8)


def k_place(P, D):
    """(byte in the head's block, shift) of each [token of a page][channel]."""
    t, c = np.meshgrid(np.arange(P), np.arange(D), indexing="ij")
    nib = np.where(c % 2 == 0, c % 8 // 2, 4 + c % 8 // 2)
    return t * (padded(D) // 2) + c // 8 * 4 + nib // 2, 4 * (nib % 2)


def v_place(P, D):
    DP = padded(D)
    t, c = np.meshgrid(np.arange(P), np.arange(D), indexing="ij")
    unit, r = c // (DP // 16), c % (DP // 16)
    byte = P * DP // 2 + t // 8 * (8 * DP // 2) + ((unit * (DP // 64) + r // 4) * 8 + t % 8) * 2 + r % 4 // 2
    return byte, 4 * (r % 2)


def quantize(x):
    """codes, scales and zero points of f32 vectors [..., D], in f32 arithmetic."""
    x = np.asarray(x, np.float32)
    x = np.where(np.isnan(x), np.float32(0), np.clip(x, np.float32(-2.0**126), np.float32(2.0**126)))
    lo, hi = np.minimum(x.min(-1), np.float32(0)), np.maximum(x.max(-1), np.float32(0))
    s = ((hi - lo) / np.float32(15)).astype(np.float32)
    s = ((s.view(np.uint32) + np.uint32(255)) & np.uint32(0xffffff00)).view(np.float32)
    d = np.where(s > 0, s, np.float32(1))
    z = np.minimum(np.rint(-lo / d), np.float32(15))
    c = np.clip(np.rint(x / d[..., None]) + z[..., None], 0, 15)
    return c.astype(np.uint8), s, z.astype(np.uint8)


class Cache:
    """The bytes of a cache, and the real values of its slots."""

    def __init__(self, pages, P, H, D, fill=0xff):
        # 0xff: records that nothing has been written to are NaN scales
        self.pages, self.P, self.H, self.D = pages, P, H, D
        self.data = np.full((pages, page_bytes(P, H, D)), fill, np.uint8)

    def block(self):
        return self.data.reshape(self.pages, self.H, -1)

    def write(self, slot, h, kind, code, scale, zero):
        """One vector: kind 0 K, 1 V."""
        byte, shift = (k_place, v_place)[kind](self.P, self.D)
        p, t = divmod(int(slot), self.P)
        b = self.block()[p, h]
        for c in range(self.D):
            at, sh = byte[t, c], int(shift[t, c])
            b[at] = (int(b[at]) & ~(15 << sh) & 255) | int(code[c]) << sh
        rec = int(np.float32(scale).view(np.uint32)) | int(zero)
        at = self.P * padded(self.D) + 4 * self.P * kind + 4 * t
        b[at:at + 4] = np.frombuffer(np.uint32(rec).tobytes(), np.uint8)

    def fill_random(self, slots, rng, k_scale=0.3, v_scale=0.1):
        """Random codes and records at the slots, all at once."""
        slots = np.asarray(slots)
        n, b = slots.size, self.block()
        p, t = slots // self.P, slots % self.P
        for h in range(self.H):
            for kind, mean in ((0, k_scale), (1, v_scale)):
                code = rng.integers(0, 16, (n, self.D))
                byte, shift = (k_place, v_place)[kind](self.P, self.D)
                for s in (0, 4):
                    r, c = np.nonzero(shift[t] == s)
                    at = byte[t][r, c]
                    keep = b[p[r], h, at] & (240 if s == 0 else 15)
                    b[p[r], h, at] = keep | (code[r, c] << s).astype(np.uint8)
                scale = (mean * np.exp(rng.normal(0, 0.5, n))).astype(np.float32)
                rec = (scale.view(np.uint32) & np.uint32(0xffffff00)) | rng.integers(0, 16, n).astype(np.uint32)
                at = self.P * padded(self.D) + 4 * self.P * kind + 4 * t
                raw = rec.astype("<u4").view(np.uint8).reshape(n, 4)
                for j in range(4):
                    b[p, h, at + j] = raw[:, j]

    def read(self, slots, h, kind):
        """Values [slots][D] in float64, and the scales."""
        slots = np.asarray(slots, np.int64)
        byte, shift = (k_place, v_place)[kind](self.P, self.D)
        p, t = slots // self.P, slots % self.P
        b = self.block()[p, h]
        code = (np.take_along_axis(b, byte[t], 1) >> shift[t]) & 15
        at = self.P * padded(self.D) + 4 * self.P * kind + 4 * t
        rec = sum(b[np.arange(slots.size), at + j].astype(np.uint32) << np.uint32(8 * j) for j in range(4))
        scale = (rec & np.uint32(0xffffff00)).view(np.float32).astype(np.float64)
        return (code - (rec & np.uint32(255)).astype(np.float64)[:, None]) * scale[:, None], scale


def attention(q, cache, table, ctx, cu, scale, causal=True, window=0):
    """q [T][Hq][D] float64.  Returns the output, and for each value how far the
    kernel's f32 sums, f16 weights and exponentials may leave it from that."""
    T, Hq, D = q.shape
    G = Hq // cache.H
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    rows = np.zeros(T, bool)
    W = table.shape[1]
    for b in range(len(ctx)):
        a, e = int(cu[b]), int(cu[b + 1])
        rows[a:e] = True
        held = min(int(ctx[b]), W * cache.P)
        page = table[b, np.arange(held) // cache.P].astype(np.int64)
        good = (page >= 0) & (page < cache.pages)
        slots = np.where(good, page, 0) * cache.P + np.arange(held) % cache.P
        tok = np.arange(held)
        for h in range(cache.H if held else 0):
            ks, ksc = cache.read(slots, h, 0)
            vs, vsc = cache.read(slots, h, 1)
            ks, vs, ksc, vsc = (np.where(good.reshape((-1,) + (1,) * (x.ndim - 1)), x, 0) for x in (ks, vs, ksc, vsc))
            for i in range(a, e):
                pos = int(ctx[b]) - (e - a) + i - a
                see = good & (tok <= pos if causal else True)
                if window:
                    see = see & (tok > pos - window)
                if not see.any():
                    continue
                # tokens that are not seen may hold anything
                k, v, sk, sv = ks[see], vs[see], ksc[see], vsc[see]
                for j in range(h * G, (h + 1) * G):
                    x = k @ q[i, j] * scale
                    p = np.exp(x - x.max())
                    total = p.sum()
                    out[i, j] = p @ v / total
                    # scores: f32 sums of D products of codes up to 15 (and of the zero
                    # point's term, as large), and a few roundings of the score itself
                    d = abs(scale) * sk * 2 * 15 * np.abs(q[i, j]).sum() * (D + 4) * 2.0**-24 + np.abs(x) * 2.0**-21
                    # weights: half a step of f16, or of its subnormals beside a largest of
                    # 1 (values of up to 15 steps); exponentials and f32 sums 2^-20 of each term
                    size = p @ np.abs(v) / total
                    tol[i, j] = size * (2.0**-11 + 2 * d.max() + 2.0**-20 + len(x) * 2.0**-24) + \
                        15 * sv.max() * len(x) * 2.0**-25
                    # the codes' and the zero point's part are summed apart
                    tol[i, j] += (p * sv).sum() / total * 30 * len(x) * 2.0**-24
    return out, tol, rows
