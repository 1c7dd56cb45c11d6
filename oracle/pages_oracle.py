"""float64 / integer definition of the 8-bit paged cache, from include/iwdft.h's description: one token, one page, one sequence at a time.  CPU only."""
from __future__ import annotations

import math

import numpy as np

LEAST = -100


def e4m3_table() -> np.ndarray:
    """What each of the 256 bytes stands for (OCP e4m3: bias 7, no infinities, S.1111.111 is NaN)."""
    out = np.empty(256)
    for byte in range(256):
        e, m = byte >> 3 & 15, byte & 7
        v = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        if byte & 127 == 127:
            v = math.nan
        out[byte] = -v if byte & 128 else v
    return out


TABLE = e4m3_table()


def to_e4m3(x: np.ndarray) -> np.ndarray:
    """Nearest byte, ties to the even mantissa, +-448 beyond; NaN as 0x7f."""
    x = np.asarray(x, np.float64)
    grid = TABLE[:127]
    mag = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), 448.0)
    hi = np.minimum(np.searchsorted(grid, mag), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - mag, mag - grid[lo]
    byte = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    byte = np.where(grid[hi] == mag, hi, byte) | np.where(np.signbit(x), 128, 0)
    return np.where(np.isnan(x), 127, byte).astype(np.uint8)


def exponent(values: np.ndarray) -> int:
    v = np.abs(np.asarray(values, np.float64))
    v = v[np.isfinite(v)]
    top = v.max() if v.size else 0.0
    e = LEAST
    while top > math.ldexp(448.0, e):
        e += 1
    return e


class Store:
    """values and exponents as numpy arrays, [layer, page, head, K/V, ...] with the tokens of a page along one axis: raw[..., token, channel]."""

    def __init__(self, n_layers, n_pages, heads, P):
        self.P = P
        self.raw = np.zeros((n_layers, n_pages, heads, 2, P, 128), np.uint8)
        self.exponents = np.zeros((n_layers, n_pages, heads, 2), np.int32)

    def packed(self) -> np.ndarray:
        """uint8 [layers, pages, heads, 2, P * 128] in the library's order."""
        n, p, h, _, P, d = self.raw.shape
        out = np.empty((n, p, h, 2, P * d), np.uint8)
        out[:, :, :, 0] = self.raw[:, :, :, 0].reshape(n, p, h, -1)
        out[:, :, :, 1] = self.raw[:, :, :, 1].reshape(n, p, h, P // 8, 8, d).swapaxes(4, 5).reshape(n, p, h, -1)
        return out

    def unpack(self, values: np.ndarray, exponents: np.ndarray):
        n, p, h, _, P, d = self.raw.shape
        self.raw[:, :, :, 0] = values[:, :, :, 0].reshape(n, p, h, P, d)
        self.raw[:, :, :, 1] = values[:, :, :, 1].reshape(n, p, h, P // 8, d, 8).swapaxes(4, 5).reshape(n, p, h, P, d)
        self.exponents[:] = exponents

    def token(self, layer, page, head, which, place) -> np.ndarray:
        return TABLE[self.raw[layer, page, head, which, place]] * 2.0 ** float(self.exponents[layer, page, head, which])

    def write(self, k, v, slots, layer0=0):
        P, n_pages = self.P, self.raw.shape[1]
        t = 0
        while t < len(slots):
            if not 0 <= slots[t] < n_pages * P:
                t += 1
                continue
            n = 1
            while t + n < len(slots) and slots[t + n] == slots[t] + n and slots[t + n] % P:
                n += 1
            page, first = slots[t] // P, slots[t] % P
            for layer in range(k.shape[0]):
                for head in range(self.raw.shape[2]):
                    for which, x in ((0, k), (1, v)):
                        new = np.asarray(x[layer, t:t + n, head], np.float64)
                        at = (layer0 + layer, page, head, which)
                        e = exponent(new)
                        if first:
                            old = int(self.exponents[at])
                            if e > old:
                                self.raw[at][:first] = to_e4m3(TABLE[self.raw[at][:first]] * 2.0 ** float(old - e))
                            e = max(e, old)
                        self.raw[at][first:first + n] = to_e4m3(new * 2.0 ** float(-e))
                        self.exponents[at] = e
            t += n

    def sequence(self, layer, head, which, pages, length) -> np.ndarray:
        """[length, 128]; NaN rows in the place of tokens whose page is not there."""
        out = np.full((length, 128), np.nan)
        for j in range(length):
            page = pages[j // self.P]
            if 0 <= page < self.raw.shape[1]:
                out[j] = self.token(layer, page, head, which, j % self.P)
        return out

    def read(self, table, lens, n, layer0, n_layers):
        """K, V [layers, batch, heads, n, 128], 0 where nothing is."""
        out = np.zeros((2, n_layers, len(lens), self.raw.shape[2], n, 128))
        for i in np.ndindex(out.shape[:4]):
            which, layer, b, head = i
            m = min(n, max(0, min(lens[b], table.shape[1] * self.P)))
            for j in range(m):
                page = table[b][j // self.P]
                if 0 <= page < self.raw.shape[1]:
                    out[i][j] = self.token(layer0 + layer, page, head, which, j % self.P)
        return out

    def attend(self, q, starts, table, lens, layer0=0, n_sink=0, n_recent=0, scale=None):
        """out [layers, rows, query heads, 128], NaN in rows of no sequence, and what bounds a computation's error: sum_j p_j |v_j| of every output, for every row
        the largest sum_i |q_i k_ij| * scale of a token it sees and the number of tokens it sees, and of every output 2^e* sum_j |v_j| 2^-e_j, e_j the
        exponent of j's page, e* that of the token with the largest p_j 2^e_j."""
        L, T, Hq, _ = q.shape
        G = Hq // self.raw.shape[2]
        scale = 1.0 / math.sqrt(128.0) if scale is None else scale
        out, weight = np.full(q.shape, np.nan), np.zeros(q.shape)
        reach, seen, floor = np.zeros(q.shape[:3]), np.zeros(q.shape[:3]), np.zeros(q.shape)
        for layer in range(L):
            for b in range(len(lens)):
                n = int(lens[b])
                for hk in range(self.raw.shape[2]):
                    k, v = (self.sequence(layer0 + layer, hk, w, table[b], n) for w in (0, 1))
                    there = np.array([0 <= table[b][j // self.P] < self.raw.shape[1] for j in range(n)], bool)
                    e = np.array([self.exponents[layer0 + layer, table[b][j // self.P], hk, 1] if there[j] else 0 for j in range(n)], np.float64)
                    j = np.arange(n)
                    for t in range(starts[b], starts[b + 1]):
                        p = n - (starts[b + 1] - starts[b]) + (t - starts[b])
                        see = there & (j <= p)
                        if n_recent:
                            see &= (j < n_sink) | (j > p - n_recent)
                        for g in range(G):
                            h = hk * G + g
                            if not see.any():
                                out[layer, t, h] = 0.0
                                continue
                            x = np.asarray(q[layer, t, h], np.float64)
                            with np.errstate(invalid="ignore"):
                                s = (k[see] @ x) * scale
                                w = np.exp(s - s.max())
                                w /= w.sum()
                                out[layer, t, h] = w @ v[see]
                                weight[layer, t, h] = w @ np.abs(v[see])
                                reach[layer, t, h] = (np.abs(k[see]) @ np.abs(x)).max() * scale
                                top = e[see][np.nanargmax(s / math.log(2.0) + e[see])] if not np.isnan(s).all() else 0.0
                                floor[layer, t, h] = (np.abs(v[see]) * 2.0 ** (top - e[see])[:, None]).sum(0)
                            seen[layer, t, h] = see.sum()
        return out, weight, reach, seen, floor


def resize(want, table, lens, free, n_slots, P):
    """In place on numpy arrays; returns starts, slots."""
    B, W = table.shape
    n_pages = len(free) - 1
    pages = lambda n: -(-n // P)  # noqa: E731
    have = [min(max(int(n), 0), W * P) for n in lens]
    want = [h if w < 0 or w > W * P else int(w) for h, w in zip(have, want)]
    stack = [int(x) for x in free[1:1 + free[0]]]
    back = [int(table[b, j]) for b in reversed(range(B)) for j in reversed(range(pages(want[b]), pages(have[b])))]  # only of shorter ones
    all_pages = stack + back
    asked = fresh = 0
    starts, slots = [0], []
    for b in range(B):
        if want[b] <= have[b]:
            lens[b] = want[b]
            starts.append(len(slots))
            continue
        need, new = pages(want[b]) - pages(have[b]), want[b] - have[b]
        asked, fresh = asked + need, fresh + new
        if fresh <= n_slots and (need == 0 or asked <= len(stack) + len(back)):
            for j in range(pages(have[b]), pages(want[b])):
                table[b, j] = all_pages.pop()
            for pos in range(have[b], want[b]):
                page = int(table[b, pos // P])
                slots.append(page * P + pos % P if 0 <= page < n_pages else -1)
            lens[b] = want[b]
        else:
            lens[b] = have[b]
        starts.append(len(slots))
    free[0] = len(all_pages)
    for i in range(len(stack), len(all_pages)):
        free[1 + i] = all_pages[i]
    slots += [-1] * (n_slots - len(slots))
    return np.array(starts, np.int32), np.array(slots, np.int32)
