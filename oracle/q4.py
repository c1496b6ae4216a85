"""The 4-bit K/V cache and 4-bit weights from their definitions, in numpy.

Nothing here is shared with the CUDA library: codes are encoded with float32
scalars as the definition states them, everything else is float64.
"""
from __future__ import annotations

import numpy as np

PAGE, GROUP = 64, 64


def encode(x):
    """One group (64 float32 values) -> (codes uint8 [64], param uint16)."""
    x = np.asarray(x, np.float32)
    if not np.all(np.isfinite(x)):
        return np.zeros(GROUP, np.uint8), np.uint16(0x7FF0)
    lo, hi = np.float32(min(0.0, x.min())), np.float32(max(0.0, x.max()))
    with np.errstate(over="ignore"):
        h = np.float16(np.float32(np.float32(hi - lo) / np.float32(15)))
    bits = (int(h.view(np.uint16)) + 15) & 0xFFF0
    if bits >= 0x7C00:
        return np.zeros(GROUP, np.uint8), np.uint16(0x7FF0)
    s = np.float32(np.uint16(bits).view(np.float16))
    if s == 0:
        z = np.float32(0)
        return np.clip(np.rint(x) + z, 0, 15).astype(np.uint8), np.uint16(0)
    z = np.clip(np.rint(np.float32(-lo) / s), 0, 15).astype(np.float32)
    if float(s) * max(z, 15 - z) > 65504:
        return np.zeros(GROUP, np.uint8), np.uint16(0x7FF0)
    return np.clip(np.rint(x / s) + z, 0, 15).astype(np.uint8), np.uint16(bits | int(z))


def decode(codes, param):
    """codes [.., 64], param [..] -> float64 values."""
    param = np.asarray(param, np.uint16)
    s = (param & 0xFFF0).astype(np.uint16).view(np.float16).astype(np.float64)
    return s[..., None] * (np.asarray(codes, np.float64) - (param & 15).astype(np.float64)[..., None])


def block_bytes(D):
    return PAGE * D + 4 * (D // GROUP) * PAGE


def block_values(block, D):
    """One block's bytes -> (K, V) float64 [64][D]."""
    block = np.asarray(block, np.uint8)
    half, G = PAGE * D // 2, D // GROUP
    out = []
    for i in range(2):
        raw = block[i * half:(i + 1) * half].reshape(PAGE, D // 2)
        codes = np.stack([raw & 15, raw >> 4], -1).reshape(PAGE, G, GROUP)
        p = block[2 * half + i * G * PAGE * 2:][:G * PAGE * 2].copy().view(np.uint16).reshape(G, PAGE).T
        out.append(decode(codes, p).reshape(PAGE, D))
    return out


def store(block, D, offset, k, v):
    """Writes one token's k, v [D] into a block's bytes at `offset`."""
    half, G = PAGE * D // 2, D // GROUP
    for i, x in enumerate((k, v)):
        for g in range(G):
            codes, param = encode(x[g * GROUP:(g + 1) * GROUP])
            at = i * half + offset * (D // 2) + g * (GROUP // 2)
            block[at:at + GROUP // 2] = codes[0::2] | codes[1::2] << 4
            at = 2 * half + (i * G * PAGE + g * PAGE + offset) * 2
            block[at:at + 2] = np.array([param], np.uint16).view(np.uint8)


def sequence(data, table, length, slot, layer, head, D):
    """K, V float64 [length][D] of one sequence's head."""
    n = int(length[slot])
    K, V = np.zeros((0, D)), np.zeros((0, D))
    parts = [block_values(data[layer, table[slot, i], head], D) for i in range(-(-n // PAGE))]
    if parts:
        K, V = (np.concatenate([p[j] for p in parts])[:n] for j in range(2))
    return K, V


def attention(q, K, V, first, scale, causal=True, window=0):
    """q [n][D] at positions first .. of a sequence with K, V [L][D].  Returns
    (out [n][D], lse [n], weight [n][D] = sum p |v|, reach [n] = the largest
    scale * sum |q k| among what a row sees)."""
    n, L, D = q.shape[0], K.shape[0], q.shape[1]
    out, lse, wt, reach = np.zeros((n, D)), np.full(n, -np.inf), np.zeros((n, D)), np.zeros(n)
    j = np.arange(L)
    for i in range(n):
        pos = first + i
        see = np.ones(L, bool)
        if causal:
            see &= j <= pos
            if window > 0:
                see &= j > pos - window
        if pos < 0 and causal or not see.any():
            continue
        a = scale * (K[see] @ q[i])
        m = a.max()
        e = np.exp(a - m)
        out[i], wt[i] = e @ V[see] / e.sum(), e @ np.abs(V[see]) / e.sum()
        lse[i] = m + np.log(e.sum())
        reach[i] = (abs(scale) * (np.abs(K[see]) @ np.abs(q[i]))).max()
    return out, lse, wt, reach


# ------------------------------------------------------------------ pages
class Pages:
    """table, length, refs as host arrays, with the upkeep's rules."""

    def __init__(self, table, length, refs):
        self.table, self.length, self.refs = table.copy(), length.copy(), refs.copy()
        self.copies = []  # (from, to) pages of the last call

    def extend(self, slots, counts):
        """Returns (indptr, where), or None where the call changes nothing."""
        self.copies = []
        S, room = len(self.length), self.table.shape[1] * PAGE
        if len(set(slots)) < len(slots) or any(not 0 <= s < S for s in slots) or any(c < 0 for c in counts):
            return None
        if any(self.length[s] + c > room for s, c in zip(slots, counts)):
            return None
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        shared = self.refs.copy()
        plan, at = [], 0
        for s, c in zip(slots, counts):
            L = int(self.length[s])
            copy = c > 0 and L % PAGE != 0 and shared[self.table[s, L // PAGE]] > 1
            new = -(-(L + c) // PAGE) - -(-L // PAGE)
            plan.append((s, c, L, copy, free[at:at + new + copy]))
            at += new + copy
        if at > len(free):
            return None
        where = []
        for s, c, L, copy, pages in plan:
            for p in pages:
                self.refs[p] = 1
            if copy:
                old = int(self.table[s, L // PAGE])
                self.refs[old] -= 1
                self.copies.append((old, pages[0]))
                self.table[s, L // PAGE], pages = pages[0], pages[1:]
            for i, p in enumerate(pages):
                self.table[s, -(-L // PAGE) + i] = p
            self.length[s] = L + c
            where += [int(self.table[s, t // PAGE]) * PAGE + t % PAGE for t in range(L, L + c)]
        return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), np.array(where, np.int32)

    def fork(self, src, dst):
        S = len(self.length)
        for i, (a, b) in enumerate(zip(src, dst)):
            others = [d for j, d in enumerate(dst) if j != i]
            if not (0 <= a < S and 0 <= b < S) or b in others or b in src or a in dst or self.length[b]:
                continue
            n = -(-int(self.length[a]) // PAGE)
            self.table[b, :n], self.length[b] = self.table[a, :n], self.length[a]
            for p in self.table[a, :n]:
                self.refs[p] += 1

    def free(self, slots, keep=None):
        for i, s in enumerate(slots):
            k = 0 if keep is None else keep[i]
            if not 0 <= s < len(self.length) or list(slots).count(s) > 1 or k < 0:
                continue
            L = int(self.length[s])
            k = min(k, L)
            for j in range(-(-k // PAGE), -(-L // PAGE)):
                self.refs[self.table[s, j]] -= 1
                self.table[s, j] = -1
            self.length[s] = k

    def compact(self):
        """Returns (table, refs, remap, live); copies holds the moves."""
        used = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        n = len(used)
        holes = [p for p in range(n) if self.refs[p] <= 0]
        self.copies = list(zip([p for p in used if p >= n], holes))
        remap = np.full(len(self.refs), -1, np.int32)
        remap[used] = used
        for a, b in self.copies:
            remap[a] = b
        table, refs = np.full_like(self.table, -1), np.zeros_like(self.refs)
        for s in range(len(self.length)):
            for j in range(-(-int(self.length[s]) // PAGE)):
                table[s, j] = remap[self.table[s, j]]
        for p in used:
            refs[remap[p]] = self.refs[p]
        return table, refs, remap, n


# ---------------------------------------------------------- 4-bit weights
def w4_values(codes, scale, minimum):
    """float64 W [N][K] from codes [N][K], scale and minimum fp16 [N][K / 128]."""
    s, m = (np.repeat(np.asarray(a, np.float16).astype(np.float64), 128, 1) for a in (scale, minimum))
    return s * np.asarray(codes, np.float64) + m


def w4_quantize(W):
    """fp16 W [N][K] -> (codes, scale, minimum) by rounding to nearest."""
    N, K = W.shape
    x = np.asarray(W, np.float16).astype(np.float32).reshape(N, K // 128, 128)
    lo, hi = x.min(-1), x.max(-1)
    s = ((hi - lo) / np.float32(15)).astype(np.float16)
    sf = s.astype(np.float32)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.clip(np.rint((x - lo[..., None]) / sf[..., None]), 0, 15)
    c = np.where(sf[..., None] > 0, c, 0)
    return c.astype(np.uint8).reshape(N, K), s, lo.astype(np.float16)
