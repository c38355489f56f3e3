"""The 8-bit paged cache in plain numpy and 64 bits, from its definition: codes, pages and attention, one number after another."""
import math

import numpy as np

INT8, E4M3 = 0, 1
SCALE_MIN, SCALE_MAX = 2.0 ** -64, 2.0 ** 64


def _e4m3_table():
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = -v if c & 128 else v
    return out


E4M3_VALUES = _e4m3_table()      # 0x7f and 0xff (NaN in the format) read as +-480: no page holds them before its length


def decode(fmt, codes):
    return codes.view(np.int8).astype(np.float64) if fmt == INT8 else E4M3_VALUES[codes]


def encode(fmt, y):
    """Codes of y (float64): nearest, half to even, saturated, 0 for NaN."""
    y = np.where(np.isnan(y), 0.0, y)
    if fmt == INT8:
        return np.clip(np.rint(np.clip(y, -1e6, 1e6)), -127, 127).astype(np.int8).view(np.uint8)
    a = np.minimum(np.abs(y), 448.0)
    e = np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -30))), -6.0)
    e = np.where((a < 2.0 ** e) & (e > -6), e - 1, e)
    a = np.minimum(np.rint(a / 2.0 ** (e - 3)) * 2.0 ** (e - 3), 448.0)
    return np.where(np.signbit(y), 128, 0).astype(np.uint8) + np.searchsorted(E4M3_VALUES[:127], a).astype(np.uint8)


def scale_of(fmt, a):
    if fmt == INT8:
        s = float(np.float32(a / 127.0)) if a / 127.0 > 1e-38 else 0.0
    else:
        s = 0.0
        if a > 0:
            e = math.frexp(a / 448.0)[1] - 2
            while 448.0 * 2.0 ** e < a:
                e += 1
            s = 2.0 ** e
    return min(max(s, SCALE_MIN), SCALE_MAX)


class Model:
    """The state of a cache and what each call makes of it.  flags: what the calls raise."""
    NO_PAGE, TOO_LONG, BAD_SEQ, BAD_PAGE = 1, 2, 4, 8

    def __init__(self, layers, num_pages, heads, page, d, fmt, max_seqs, max_pages):
        self.fmt, self.page, self.heads, self.d = fmt, page, heads, d
        self.code = [np.zeros((layers, num_pages, heads, page, d), np.uint8) for _ in range(2)]
        self.scale = [np.ones((layers, num_pages, heads)) for _ in range(2)]
        self.table = np.full((max_seqs, max_pages), -1, np.int64)
        self.lengths = np.zeros(max_seqs, np.int64)
        self.refs = np.zeros(num_pages, np.int64)
        self.flags = 0

    def _free_pages(self):
        return [int(p) for p in np.flatnonzero(self.refs == 0)]

    def reserve(self, seqs, add):
        first, free, stuck, seen = [], self._free_pages(), False, set()
        for s, a in zip(seqs, add):
            first.append(-1)
            if s == -1:
                continue
            if not 0 <= s < len(self.lengths) or s in seen or a < 0:
                self.flags |= self.BAD_SEQ
                seen.add(s)
                continue
            seen.add(s)
            old, new = int(self.lengths[s]), int(self.lengths[s]) + a
            if new > self.table.shape[1] * self.page:
                self.flags |= self.TOO_LONG
                continue
            have, want = -(-old // self.page), -(-new // self.page)
            if want > have and (stuck or want - have > len(free)):
                stuck = True
                self.flags |= self.NO_PAGE
                continue
            for col in range(have, want):
                p = free.pop(0)
                self.table[s, col], self.refs[p] = p, 1
            self.lengths[s] = new
            first[-1] = old
        return first

    def store(self, layer, k, v, seqs, first, cu):
        for which, x in ((0, k), (1, v)):
            code, scale = self.code[which][layer], self.scale[which][layer]
            for i, s in enumerate(seqs):
                if s == -1 or first[i] < 0:
                    continue
                t, pos = cu[i], first[i]
                while t < cu[i + 1]:
                    slot = pos % self.page
                    m = min(self.page - slot, cu[i + 1] - t)
                    p = self.table[s, pos // self.page]
                    for h in range(self.heads):
                        new = x[t:t + m, h].astype(np.float64)
                        fin = np.abs(new[np.isfinite(new)])
                        sc = scale_of(self.fmt, float(fin.max()) if fin.size else 0.0)
                        if slot:
                            old = scale[p, h]
                            sc = max(sc, old)
                            if sc > old:
                                code[p, h, :slot] = encode(self.fmt, decode(self.fmt, code[p, h, :slot]) * old / sc)
                        scale[p, h] = sc
                        with np.errstate(over="ignore", invalid="ignore"):
                            code[p, h, slot:slot + m] = encode(self.fmt, new / sc)
                    t, pos = t + m, pos + m

    def rows(self, layer, which, s):
        """[heads][length][d] values of a sequence."""
        n = int(self.lengths[s])
        pages = self.table[s, : -(-n // self.page)]
        x = decode(self.fmt, self.code[which][layer][pages]) * self.scale[which][layer][pages][..., None, None]
        return x.transpose(1, 0, 2, 3).reshape(self.heads, -1, self.d)[:, :n]

    def attend(self, layer, q, seqs, cu, scale, causal=True, window=0):
        """(out, lse, size, reach, tiny): also, for error bounds, sum_j w_j |v_j| per channel, the largest sum_c |q_c k_jc| scale of a row, and the
        tokens that it sees times the largest product of a weight and its value's scale."""
        total, H, d = q.shape
        G = H // self.heads
        out, lse = np.zeros((total, H, d)), np.full((total, H), -np.inf)
        size, reach, tiny = np.zeros((total, H, d)), np.zeros((total, H)), np.zeros((total, H))
        for i, s in enumerate(seqs):
            m = cu[i + 1] - cu[i]
            if s == -1 or m == 0:
                continue
            n = int(self.lengths[s])
            K, V = self.rows(layer, 0, s), self.rows(layer, 1, s)
            j = np.arange(n)
            pages = self.table[s, : -(-n // self.page)]
            vs = np.repeat(self.scale[1][layer][pages], self.page, axis=0)[:n].T
            for t in range(m):
                p = n - m + t
                seen = j <= p if causal else j >= 0
                if window:
                    seen &= j > p - window
                if not seen.any():
                    continue
                for h in range(H):
                    kk, vv = K[h // G][seen], V[h // G][seen]
                    qq = q[cu[i] + t, h].astype(np.float64)
                    x = kk @ qq * scale
                    w = np.exp(x - x.max())
                    lse[cu[i] + t, h] = x.max() + math.log(w.sum())
                    w /= w.sum()
                    out[cu[i] + t, h], size[cu[i] + t, h] = w @ vv, w @ np.abs(vv)
                    reach[cu[i] + t, h] = (np.abs(kk) @ np.abs(qq)).max() * abs(scale)
                    tiny[cu[i] + t, h] = w.size * (w * vs[h // G][seen]).max()
        return out, lse, size, reach, tiny

    def fork(self, src, dst):
        lengths, free, stuck, seen = self.lengths.copy(), self._free_pages(), False, set()
        for a, b in zip(src, dst):
            if a == -1 or b == -1:
                continue
            if not 0 <= b < len(lengths) or b in seen or not 0 <= a < len(lengths) or lengths[b]:
                self.flags |= self.BAD_SEQ
                seen.add(b)
                continue
            seen.add(b)
            n = int(lengths[a])
            full = n // self.page
            if n % self.page:
                if stuck or not free:
                    stuck = True
                    self.flags |= self.NO_PAGE
                    continue
                p = free.pop(0)
                for x in self.code + self.scale:
                    x[:, p] = x[:, self.table[a, full]]
                self.table[b, full], self.refs[p] = p, 1
            self.table[b, :full] = self.table[a, :full]
            np.add.at(self.refs, self.table[a, :full], 1)
            self.lengths[b] = n

    def free(self, seqs):
        seen = set()
        for s in seqs:
            if s == -1:
                continue
            if not 0 <= s < len(self.lengths) or s in seen:
                self.flags |= self.BAD_SEQ
                continue
            seen.add(s)
            np.add.at(self.refs, self.table[s][self.table[s] >= 0], -1)
            self.table[s], self.lengths[s] = -1, 0

    def compact(self):
        used = int((self.refs > 0).sum())
        to = [p for p in range(used) if self.refs[p] == 0]
        of = [p for p in range(used, len(self.refs)) if self.refs[p] > 0]
        remap = np.where(self.refs > 0, np.arange(len(self.refs)), -1)
        remap[of] = to
        for x in self.code + self.scale:
            x[:, to] = x[:, of]
        self.refs[to], self.refs[of] = self.refs[of], 0
        self.table = np.where(self.table >= 0, remap[self.table], -1)
        return remap
