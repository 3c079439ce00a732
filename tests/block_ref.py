"""Plain 64-bit forms of the block-scaled cache, one sequence at a time, and inputs for them."""
import math

import numpy as np
import torch

PAGE = 128


def e4m3_values():
    v = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[code] = math.nan if code & 127 == 127 else -x if code >> 7 else x
    return v


VALUES = e4m3_values()


def encode(x):
    """Nearest code, ties to the even one, 448 at most; NaN: 0x7f."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    a = np.where(np.isnan(x), 0.0, a)
    hi = np.clip(np.searchsorted(VALUES[:127], a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - VALUES[lo], VALUES[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(np.isnan(x), 0x7f, code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def needed(x):
    """x [n][Hkv][D]: per head the smallest 2^e, e >= -100, with amax <= 448 * 2^e over finite entries."""
    x = np.where(np.isfinite(x), np.abs(x), 0.0)
    top = x.max(axis=(0, 2))
    out = np.empty(len(top))
    for h, t in enumerate(top):
        e = -100
        while 448.0 * 2.0 ** e < t:
            e += 1
        out[h] = 2.0 ** e
    return out


class Cache:
    """One layer's K or V: codes [pages * 128][Hkv][D] uint8, scales [pages][Hkv][128 / block]."""

    def __init__(self, codes, scales, block, table):
        self.codes, self.scales, self.block, self.table = codes, scales, block, table

    def slot(self, b, p):
        return int(self.table[b, p // PAGE]) * PAGE + p % PAGE

    def scale(self, b, p):
        return self.scales[int(self.table[b, p // PAGE]), :, p % PAGE // self.block]

    def read(self, b, positions):
        """[n][Hkv][D] values"""
        return np.stack([VALUES[self.codes[self.slot(b, p)]] * self.scale(b, p)[:, None].astype(np.float64) for p in positions])

    def _put(self, b, positions, x, kept, fresh):
        for j in sorted({p // self.block for p in positions}):
            mine = [i for i, p in enumerate(positions) if p // self.block == j]
            stay = [p for p in kept if p // self.block == j]
            was = self.scale(b, j * self.block).astype(np.float64).copy()
            now = needed(x[mine]) if fresh and not stay else np.maximum(was, needed(x[mine]))
            grown = now > was
            for p in stay:
                if grown.any():
                    again = encode(VALUES[self.codes[self.slot(b, p)]] * was[:, None] / now[:, None])
                    self.codes[self.slot(b, p)][grown] = again[grown]
            for i in mine:
                self.codes[self.slot(b, positions[i])] = encode(x[i] / now[:, None])
            self.scale(b, j * self.block)[:] = now

    def append(self, b, P, rows):
        first = P // self.block * self.block
        self._put(b, [P + i for i in range(len(rows))], rows, range(first, P), True)

    def compact(self, b, P, a, path):
        if a == 0:
            return
        x = self.read(b, [P + int(path[i]) for i in range(1, a + 1)])
        first = P // self.block * self.block
        self._put(b, [P + i for i in range(1, a + 1)], x, range(first, P + 1), False)


def pages(lengths, r, spare=3, extra=1):
    need = [-(-int(n) // PAGE) for n in lengths]
    n = sum(need) + spare
    perm, at = r.permutation(n), 0
    table = np.full((len(need), max(max(need), 1) + extra), -1, np.int32)
    for b, k in enumerate(need):
        table[b, :k] = perm[at:at + k]
        at += k
    return n, table


def tree(r, B, T, C):
    parent = np.full((B, T), -1, np.int32)
    for i in range(1, T):
        parent[:, i] = r.randint(max(0, i - 4), i, B)
    owner = np.sort(r.randint(0, T, (B, C)), axis=1).astype(np.int32)
    return parent, owner


def visible(P, T, C, S, parent, owner):
    """[R][P + R + S]"""
    R = T + C
    see = np.zeros((R, P + R + S), bool)
    see[:, :P] = True
    for i in range(R):
        node = i if i < T else int(owner[i - T])
        see[i, P + i] = True
        while node >= 0:
            see[i, P + node] = True
            node = int(parent[node])
        see[i, P + R:] = i >= T
    return see


def attention(q, k, v, v_scale, see, sm_scale, weight_bits):
    """q [R][Hq][D], k, v [n][Hkv][D] values, v_scale [n][Hkv] their scales: (out, lse, tolerance of out, of lse), 64 bits.

    Tolerance of an element, beyond the rounding of the output to bf16 (2^-8 of it):
      a weight rounded to `weight_bits` bits                      2^-weight_bits of sum w |v|
      scores: fp32 sums of D exact products, then products with factors and a sum with the maximum, all fp32, and the exponential's
      own error (2^-22): 2 (numerator and denominator) times  D 2^-24 max sum |q k| c  +  2^-22 (max |s| + |log2 v scale| + 8)
      a weight times V scale that is smaller than 2^-14 of the largest keeps 2^-25 of that:  sum 2^-25 |code| max(w v_scale), over l
    lse: the same error of the scores, and fp32 rounding of the result."""
    R, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    out, tol = np.zeros((R, Hq, D)), np.zeros((R, Hq, D))
    lse, tol_lse = np.zeros((R, Hq)), np.zeros((R, Hq))
    for h in range(Hq):
        g = h // G
        anywhere = see.any(0)
        kk, vv = np.where(anywhere[:, None], k[:, g], 0.0), np.where(anywhere[:, None], v[:, g], 0.0)
        vs = np.where(anywhere, v_scale[:, g], 1.0)
        s = q[:, h] @ kk.T * sm_scale
        s = np.where(see, s, -np.inf)
        top = s.max(1, keepdims=True)
        w = np.exp(s - top)
        l = w.sum(1, keepdims=True)
        out[:, h] = w @ vv / l
        lse[:, h] = (top + np.log(l))[:, 0]
        mag = (np.abs(q[:, h]) @ np.abs(kk).T * sm_scale * see).max(1, keepdims=True)
        score = D * 2.0 ** -24 * mag + 2.0 ** -22 * (mag + np.abs(np.log2(vs)).max() + 8)
        weighted = w @ np.abs(vv) / l
        low = 2.0 ** -25 * (w * vs).max(1, keepdims=True) * 256 * (see @ np.abs(vv / vs[:, None])) / l
        tol[:, h] = 2.0 ** -8 * np.abs(out[:, h]) + (2.0 ** -weight_bits + 2 * score) * weighted + low + 2.0 ** -133
        tol_lse[:, h] = (score + 2.0 ** -22 * (1 + np.abs(lse[:, h:h + 1])))[:, 0]
    return out, lse, tol, tol_lse


def to_cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()
