"""Float64 definitions of the paged-cache operators, in NumPy, on the host.

Written from the formulas and from what the operators promise, one stream and
one page at a time; shares no code with the GPU path.
"""

import math

import numpy as np


# ------------------------------------------------------------------ rotation
def scaled_freqs(rot_dim, theta, scaling, factor=1.0, native_len=0, beta_fast=32.0,
                 beta_slow=1.0):
    """(frequencies of the rot_dim/2 pairs, factor of cos and sin)."""
    i = np.arange(rot_dim // 2, dtype=np.float64)
    f = theta ** (-2.0 * i / rot_dim)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "ntk":
        return (theta * factor ** (rot_dim / (rot_dim - 2.0))) ** (-2.0 * i / rot_dim), 1.0
    if scaling == "yarn":
        turns = native_len * f / (2.0 * math.pi)
        keep = np.clip((turns - beta_slow) / (beta_fast - beta_slow), 0.0, 1.0)
        return (1.0 - keep) * f / factor + keep * f, 1.0 + 0.1 * math.log(factor)
    return f, 1.0


def rotate(x, pos, table, pairs, offset=0, half=False, inverse=False):
    """x [tokens, heads, dim] float64, pos [tokens, axes], table [len, m, 2]."""
    y = np.array(x, dtype=np.float64)
    m = sum(pairs)
    axis = np.repeat(np.arange(3), pairs)
    for t in range(x.shape[0]):
        cs = np.asarray([table[pos[t, axis[i]], i] for i in range(m)], dtype=np.float64)
        z = cs[:, 0] + 1j * cs[:, 1] * (-1.0 if inverse else 1.0)
        part = np.asarray(x[t, :, offset:offset + 2 * m], dtype=np.float64)
        w = (part[:, :m] + 1j * part[:, m:]) if half else (part[:, 0::2] + 1j * part[:, 1::2])
        w = w * z
        if half:
            y[t, :, offset:offset + m], y[t, :, offset + m:offset + 2 * m] = w.real, w.imag
        else:
            y[t, :, offset:offset + 2 * m:2], y[t, :, offset + 1:offset + 2 * m:2] = w.real, w.imag
    return y


# --------------------------------------------------------------------- pages
class Pages:
    """Page metadata and contents, with the rules of the page operations."""

    def __init__(self, layers, pages, page_tokens, seqs, max_pages, d_c, d_r):
        self.P, self.max_pages = page_tokens, max_pages
        self.table = np.full((seqs, max_pages), -1, dtype=np.int32)
        self.lens = np.zeros(seqs, dtype=np.int32)
        self.refs = np.zeros(pages, dtype=np.int32)
        self.c = np.zeros((layers, pages, page_tokens, d_c))
        self.kr = np.zeros((layers, pages, page_tokens, d_r))
        self.range_error = False

    def _n(self, tokens):
        return -(-int(tokens) // self.P)

    def resize(self, new_lens):
        S, cap = len(self.lens), self.max_pages * self.P
        new = [int(v) for v in new_lens]
        for s in range(S):
            if new[s] > cap:
                self.range_error = True
                new[s] = -1
        for s in range(S):
            if 0 <= new[s] < self.lens[s]:
                for j in range(self._n(new[s]), self._n(self.lens[s])):
                    self.refs[self.table[s, j]] -= 1
                    self.table[s, j] = -1
                self.lens[s] = new[s]
        grow = [s for s in range(S) if new[s] > self.lens[s]]
        tail = {s: self.table[s, self._n(self.lens[s]) - 1] for s in grow if self.lens[s] % self.P}
        cow = {s for s, pg in tail.items() if self.refs[pg] > 1}
        free = [int(p) for p in np.flatnonzero(self.refs == 0)]
        at, given_back = 0, []
        for s in grow:
            have, want = self._n(self.lens[s]), self._n(new[s])
            need = want - have + (s in cow)
            got = free[at:at + need]
            at += need                     # a stream that does not fit still counts
            if len(got) < need:
                self.range_error = True
                continue
            if s in cow:
                rows, to = int(self.lens[s]) % self.P, got.pop(0)
                self.c[:, to, :rows] = self.c[:, tail[s], :rows]
                self.kr[:, to, :rows] = self.kr[:, tail[s], :rows]
                self.table[s, have - 1] = to
                self.refs[to] = 1
                given_back.append(tail[s])
            for j, p in enumerate(got):
                self.table[s, have + j] = p
                self.refs[p] = 1
            self.lens[s] = new[s]
        for p in given_back:
            self.refs[p] -= 1

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            S = len(self.lens)
            if not (0 <= a < S and 0 <= b < S) or a == b or self.lens[b]:
                self.range_error = True
                continue
            for j in range(self._n(self.lens[a])):
                self.table[b, j] = self.table[a, j]
                self.refs[self.table[a, j]] += 1
            self.lens[b] = self.lens[a]

    def compact(self):
        live = [int(p) for p in np.flatnonzero(self.refs > 0)]
        n = len(live)
        holes = [p for p in range(n) if self.refs[p] <= 0]
        for to, of in zip(holes, [p for p in live if p >= n]):
            self.c[:, to], self.kr[:, to] = self.c[:, of], self.kr[:, of]
            self.table[self.table == of] = to
            self.refs[to], self.refs[of] = self.refs[of], 0

    def append(self, layer, c_new, kr_rot, q_start):
        for s in range(len(self.lens)):
            n = q_start[s + 1] - q_start[s]
            for i in range(n):
                a = int(self.lens[s]) - n + i
                p = self.table[s, a // self.P]
                self.c[layer, p, a % self.P] = c_new[q_start[s] + i]
                self.kr[layer, p, a % self.P] = kr_rot[q_start[s] + i]

    def rows(self, layer, s):
        """(c, kr) of stream s, token after token."""
        a = np.arange(self.lens[s])
        p = self.table[s, a // self.P]
        return self.c[layer, p, a % self.P], self.kr[layer, p, a % self.P]


# ----------------------------------------------------------------- attention
def visible(place, held, block):
    """Keys that a token at `place` of a stream of `held` tokens sees."""
    if place < 0:
        return 0
    return held if block == 0 else min(held, (place // block + 1) * block)


def attend(q_c, q_r, c, kr, head_dim, block, v=None):
    """Newest tokens of one stream: q_c [n, H, d_c], q_r [n, H, d_r] rotated, c
    [held, d_c], kr [held, d_r]; a row that sees nothing is 0. float64. The weights
    multiply c, or v: |c| gives the size that rounding errors go by."""
    v = c if v is None else v
    n, held = q_c.shape[0], c.shape[0]
    out = np.zeros(q_c.shape)
    for i in range(n):
        k = visible(held - n + i, held, block)
        if k == 0:
            continue
        s = (q_c[i] @ c[:k].T + q_r[i] @ kr[:k].T) / math.sqrt(head_dim)
        w = np.exp(s - s.max(-1, keepdims=True))
        out[i] = (w / w.sum(-1, keepdims=True)) @ v[:k]
    return out
