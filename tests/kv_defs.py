"""The 8-bit key/value cache from its definition, in 64 bits on the CPU: plain
loops over sequences, blocks and heads, no code of the package."""
import math

import numpy as np

E4M3, INT8 = 0, 1
LIMIT = {E4M3: 448.0, INT8: 127.0}


def _e4m3_table():
    out = np.empty(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if b & 127 == 127:
            x = math.nan
        out[b] = -x if b > 127 else x
    return out


E4M3_VALUES = _e4m3_table()
_POSITIVE = E4M3_VALUES[:127]  # ascending, code = index


def encode(x, kind):
    """Values (already scaled, within the largest code) to codes, nearest, ties to even."""
    x = np.asarray(x, np.float64)
    if kind == INT8:
        return np.rint(x).astype(np.int8).view(np.uint8)
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    return (code + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def decode(code, kind):
    code = np.asarray(code, np.uint8)
    return E4M3_VALUES[code] if kind == E4M3 else code.view(np.int8).astype(np.float64)


def least_exponent(top, limit):
    """The least e in [-100, 120] with top <= limit * 2^e."""
    if top == 0:
        return -100
    e = math.frexp(top)[1] - math.frexp(limit)[1]
    if top > limit * 2.0 ** e:
        e += 1
    return min(120, max(-100, e))


class RefCache:
    def __init__(self, n_blocks, heads, dim, block, kind):
        self.n_blocks, self.heads, self.dim, self.block, self.kind = n_blocks, heads, dim, block, kind
        self.k_code = np.zeros((n_blocks, heads, block, dim), np.uint8)
        self.v_code = np.zeros((n_blocks, heads, dim, block), np.uint8)
        self.k_exp = np.zeros((n_blocks, heads), np.int8)
        self.v_exp = np.zeros((n_blocks, heads), np.int8)
        self.mean_code = np.zeros((n_blocks, heads, dim), np.int8)
        self.mean_exp = np.zeros((n_blocks, heads), np.int8)

    def _block(self, x, held, was):
        finite = np.abs(x[np.isfinite(x)])
        e = least_exponent(float(finite.max()) if finite.size else 0.0, LIMIT[self.kind])
        if len(held):
            e = max(e, was)
            if e > was:
                held = encode(decode(held, self.kind) * 2.0 ** (was - e), self.kind)
        y = np.where(np.isnan(x), 0.0, np.clip(x, -3.5e38, 3.5e38) * 2.0 ** -e)
        new = encode(np.clip(y, -LIMIT[self.kind], LIMIT[self.kind]), self.kind)
        return np.concatenate([held, new]), e

    def write(self, table, length, begin, k, v):
        t = self.block
        for s in range(len(length)):
            n, row = begin[s + 1] - begin[s], begin[s]
            pos, end = length[s] - n, length[s]
            while pos < end:
                b, a = pos // t, pos % t
                z = min(t, a + end - pos)
                p = table[s][b]
                for h in range(self.heads):
                    for name, x in (("k", k), ("v", v)):
                        code = getattr(self, name + "_code")[p, h]
                        code = code if name == "k" else code.T
                        exp = getattr(self, name + "_exp")
                        new, e = self._block(x[row:row + z - a, h], code[:a], int(exp[p, h]))
                        code[:z], exp[p, h] = new, e
                    if z == t:
                        total = decode(self.k_code[p, h], self.kind).sum(0)
                        top = float(np.abs(total).max())
                        e = least_exponent(top, 127.0) if top else -15
                        self.mean_code[p, h] = np.rint(total * 2.0 ** -e)
                        self.mean_exp[p, h] = int(self.k_exp[p, h]) + e - int(math.log2(t))
                row += z - a
                pos += z - a

    def values(self, pages, h):
        """Keys and values of one head of these blocks: [token, dim] each."""
        k = decode(self.k_code[pages, h], self.kind) * 2.0 ** self.k_exp[pages, h].astype(float)[:, None, None]
        v = decode(self.v_code[pages, h], self.kind) * 2.0 ** self.v_exp[pages, h].astype(float)[:, None, None]
        return k.reshape(-1, self.dim), v.transpose(0, 2, 1).reshape(-1, self.dim)

    def read(self, table, length, begin):
        k = np.zeros((begin[-1], self.heads, self.dim))
        v = np.zeros_like(k)
        for s in range(len(length)):
            n = begin[s + 1] - begin[s]
            if not n:
                continue
            for h in range(self.heads):
                ks, vs = self.values(table[s][:(length[s] + self.block - 1) // self.block], h)
                k[begin[s]:begin[s + 1], h] = ks[length[s] - n:length[s]]
                v[begin[s]:begin[s + 1], h] = vs[length[s] - n:length[s]]
        return k, v

    def attend(self, table, length, begin, q, scale, blocks=None):
        """(out, lse, mass, delta, floor): mass[row, head, d] = the weighted mean of |v|, delta[row,
        head] = the largest sum of |scale q k| of a seen key, floor[row, head] = the seen places
        times the largest value that the cache's codes can hold in the sequence's blocks: what the
        error bounds are made of."""
        group = q.shape[1] // self.heads
        out = np.zeros(q.shape)
        mass = np.zeros(q.shape)
        lse = np.full(q.shape[:2], -np.inf)
        delta = np.zeros(q.shape[:2])
        floor = np.zeros(q.shape[:2])
        t = self.block
        for s in range(len(length)):
            n = begin[s + 1] - begin[s]
            for h in range(self.heads):
                if length[s] == 0 or n == 0:
                    continue
                pages = table[s][:(length[s] + t - 1) // t]
                ks, vs = self.values(pages, h)
                largest = LIMIT[self.kind] * 2.0 ** float(self.v_exp[pages, h].max())
                for i in range(n):
                    row, p = begin[s] + i, length[s] - n + i
                    if p < 0:
                        continue
                    if blocks is None:
                        seen = np.arange(p + 1)
                    else:
                        named = blocks[row, h][blocks[row, h] >= 0]
                        seen = (named[:, None] * t + np.arange(t)).reshape(-1)
                        seen = seen[seen <= p]
                        if not len(seen):
                            continue
                    for g in range(h * group, (h + 1) * group):
                        x = scale * (ks[seen] @ q[row, g])
                        top = x.max()
                        w = np.exp(x - top)
                        out[row, g] = w @ vs[seen] / w.sum()
                        mass[row, g] = w @ np.abs(vs[seen]) / w.sum()
                        lse[row, g] = top + math.log(w.sum())
                        floor[row, g] = len(seen) * largest
                        delta[row, g] = abs(scale) * (np.abs(ks[seen]) @ np.abs(q[row, g])).max()
        return out, lse, mass, delta, floor

    def select(self, table, length, begin, q, keep, first, recent):
        group, t = q.shape[1] // self.heads, self.block
        out = np.full((begin[-1], self.heads, keep), -1, np.int32)
        for s in range(len(length)):
            n = begin[s + 1] - begin[s]
            for i in range(n):
                row, p = begin[s] + i, length[s] - n + i
                nb = p // t + 1 if p >= 0 else 0
                for h in range(self.heads):
                    if nb <= keep:
                        out[row, h, :nb] = np.arange(nb)
                        continue
                    pages = table[s][:nb]
                    mean = self.mean_code[pages, h].astype(float) * 2.0 ** self.mean_exp[pages, h].astype(float)[:, None]
                    score = np.full(nb, -np.inf)
                    for g in range(h * group, (h + 1) * group):
                        x = q[row, g]
                        e = math.frexp(float(np.abs(x).max()))[1] if np.abs(x).max() > 0 else 0
                        code = np.clip(np.rint(x * 2.0 ** (7 - e)), -127, 127)
                        score = np.maximum(score, mean @ code * 2.0 ** (e - 7))
                    middle = sorted(range(first, nb - recent), key=lambda b: (-score[b], b))
                    taken = [*range(first), *middle[:keep - first - recent], *range(nb - recent, nb)]
                    out[row, h] = sorted(taken)
        return out
