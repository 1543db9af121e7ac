"""The key/value cache in 4 bits from its definition, in 64 bits on the CPU: no code of the package."""
import math

import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6])


def encode4(x):
    """Scaled values to codes, nearest, ties to even; beyond 6 is 6."""
    a = np.minimum(np.abs(x), 6.0)
    hi = np.clip(np.searchsorted(VALUES[:8], a), 1, 7)
    up, down = VALUES[hi] - a, a - VALUES[hi - 1]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return (code + np.where(np.signbit(x), 8, 0)).astype(np.uint8)


def least_exponent4(top):
    """The least e in [-100, 120] with top <= 7 * 2^e."""
    if top == 0:
        return -100
    e = math.frexp(top)[1] - 3
    if top > 7.0 * 2.0 ** e:
        e += 1
    return min(120, max(-100, e))


def quantise(x):
    """x [..., dim] to (codes [..., dim], exponents [..., dim / 32])."""
    y = x.reshape(*x.shape[:-1], -1, 32)
    finite = np.where(np.isfinite(y), np.abs(y), 0.0)
    e = np.vectorize(least_exponent4)(finite.max(-1)) if finite.size else np.zeros(y.shape[:-1], int)
    scaled = np.where(np.isnan(y), 0.0, np.clip(y, -3.5e38, 3.5e38) * 2.0 ** -e.astype(float)[..., None])
    return encode4(scaled).reshape(x.shape), e


class RefCache4:
    def __init__(self, n_blocks, heads, dim, block):
        self.n_blocks, self.heads, self.dim, self.block = n_blocks, heads, dim, block
        self.k_code, self.v_code = (np.zeros((n_blocks, heads, block, dim // 2), np.uint8) for _ in range(2))
        self.k_exp, self.v_exp = (np.full((n_blocks, heads, dim // 32, block), 127, np.uint8) for _ in range(2))

    def write(self, table, length, begin, k, v):
        for x, code, exp in ((k, self.k_code, self.k_exp), (v, self.v_code, self.v_exp)):
            c, e = quantise(x)
            for s in range(len(length)):
                n = begin[s + 1] - begin[s]
                for i in range(n):
                    pos = length[s] - n + i
                    p, slot = table[s][pos // self.block], pos % self.block
                    row = c[begin[s] + i]
                    code[p, :, slot] = row[:, 0::2] + (row[:, 1::2] << 4)
                    exp[p, :, :, slot] = e[begin[s] + i] + 127

    def values(self, pages, h):
        """Keys and values of one head of these blocks: [token, dim] each."""
        out = []
        for code, exp in ((self.k_code, self.k_exp), (self.v_code, self.v_exp)):
            c = code[pages, h]
            x = np.stack([VALUES[c & 15], VALUES[c >> 4]], -1).reshape(*c.shape[:-1], self.dim)
            scale = 2.0 ** (exp[pages, h].astype(float) - 127.0)
            out.append((x * np.repeat(scale.transpose(0, 2, 1), 32, -1)).reshape(-1, self.dim))
        return out

    def read(self, table, length, begin):
        k = np.zeros((begin[-1], self.heads, self.dim))
        v = np.zeros_like(k)
        for s in range(len(length)):
            n = begin[s + 1] - begin[s]
            for h in range(self.heads):
                ks, vs = self.values(table[s][:(length[s] + self.block - 1) // self.block], h)
                k[begin[s]:begin[s + 1], h] = ks[length[s] - n:length[s]]
                v[begin[s]:begin[s + 1], h] = vs[length[s] - n:length[s]]
        return k, v

    def attend(self, table, length, begin, q, scale):
        """(out, lse, mass, delta, floor): mass[row, head, d] = the weighted mean of |v|, delta[row, head] = the
        largest sum of |scale q k| of a seen key, floor[row, head, d] = the sum of the seen 1 + |v|: what the error
        bounds are made of."""
        group = q.shape[1] // self.heads
        out, mass, floor = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape)
        lse, delta = np.full(q.shape[:2], -np.inf), np.zeros(q.shape[:2])
        for s in range(len(length)):
            n = begin[s + 1] - begin[s]
            if length[s] == 0 or n == 0:
                continue
            rows = slice(begin[s], begin[s + 1])
            p = length[s] - n + np.arange(n)
            for h in range(self.heads):
                ks, vs = self.values(table[s][:(length[s] + self.block - 1) // self.block], h)
                ks, vs = ks[:length[s]], vs[:length[s]]
                hide = np.arange(length[s]) > p[:, None]
                some = p >= 0
                for g in range(h * group, (h + 1) * group):
                    x = scale * (q[rows, g] @ ks.T)
                    x[hide] = -np.inf
                    top = np.where(some, x.max(1), 0.0)
                    w = np.exp(x - top[:, None])
                    total = np.where(some, w.sum(1), 1.0)
                    out[rows, g] = (w @ vs) / total[:, None]
                    mass[rows, g] = (w @ np.abs(vs)) / total[:, None]
                    floor[rows, g] = np.where(hide, 0.0, 1.0) @ (1.0 + np.abs(vs))
                    lse[rows, g] = np.where(some, top + np.log(total), -np.inf)
                    d = abs(scale) * (np.abs(q[rows, g]) @ np.abs(ks).T)
                    d[hide] = 0.0
                    delta[rows, g] = d.max(1)
        return out, lse, mass, delta, floor
