"""Rotations, trees of drafted tokens and their acceptance on the host, in 64
bits: what the tests compare the library with."""
import numpy as np

from tests.pages_model import HostPages, OK, ESEQ, ELEN, ESHARED

EPATH = 5


def frequencies(dim, base=10000.0, scaling=None, factor=1.0, original_len=4096.0, slow=1.0, fast=32.0):
    """(radians a position of each pair, amplitude) by the rules of dllm_rps.h."""
    j = np.arange(dim // 2)
    if scaling == "base" and dim > 2:
        base = base * factor ** (dim / (dim - 2))
    f = base ** (-2.0 * j / dim)
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        stay = np.clip((original_len * f / (2 * np.pi) - slow) / (fast - slow), 0, 1)
        return f * stay + f / factor * (1 - stay), 0.1 * np.log(factor) + 1
    return f, 1.0


def rotate(x, pos, freq, dim, pairs, amplitude=1.0, norm=False, gain=None, eps=1e-5):
    """x [..., heads, hd] at positions pos [...].  Returns the result and, per
    element, the sum of magnitudes that it is made of."""
    x = np.asarray(x, dtype=np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if gain is not None:
            x = x * gain
    y, mass = x.copy(), np.abs(x)
    if dim:
        a = slice(0, dim, 2) if pairs else slice(0, dim // 2)
        b = slice(1, dim, 2) if pairs else slice(dim // 2, dim)
        t = np.asarray(pos, dtype=np.float64)[..., None, None] * freq
        c, s = np.cos(t) * amplitude, np.sin(t) * amplitude
        y[..., a], y[..., b] = c * x[..., a] - s * x[..., b], s * x[..., a] + c * x[..., b]
        both = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(amplitude)
        mass[..., a], mass[..., b] = both, both
    return y, mass


def sees(parent):
    """[rows][rows]: whether row i sees row j, from each row's parent."""
    n = len(parent)
    m = np.zeros((n, n), dtype=bool)
    for i, p in enumerate(parent):
        if 0 <= p < i:
            m[i] = m[p]
        m[i, i] = True
    return m


def words(see, max_rows):
    """Bits of [rows][rows] as [rows][words] int32."""
    w = (max_rows + 31) // 32
    out = np.zeros((see.shape[0], w), dtype=np.int64)
    for j in range(see.shape[1]):
        out[:, j // 32] |= see[:, j].astype(np.int64) << (j % 32)
    return out.astype(np.uint32).view(np.int32).reshape(see.shape[0], w)


def attend_tree(q, keys, values, counts, see, scale):
    """As pages_model.attend, for the last counts[b] of the positions in a tree:
    row i sees the positions before them, and row j where see[b][i, j]."""
    n, rows, heads, hd = q.shape
    out, mass, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros((n, rows, heads, 1))
    for b in range(n):
        m, c = keys[b].shape[0], counts[b]
        if m == 0 or c == 0:
            continue
        seen = np.ones((c, m), dtype=bool)
        first = m - c
        for j in range(c):
            if first + j >= 0:
                seen[:, first + j] = see[b][:c, j]
        some = seen.any(1)
        for h in range(heads):
            kv = h // (heads // keys[b].shape[1])
            k, v = keys[b][:, kv], values[b][:, kv]
            z = np.where(seen, q[b, :c, h] @ k.T * scale, -np.inf)
            top = np.where(some[:, None], z.max(1, keepdims=True), 0.0)
            w = np.exp(z - top)
            w /= np.maximum(w.sum(1, keepdims=True), 1e-300)
            out[b, :c, h], mass[b, :c, h] = w @ v, w @ np.abs(v)
            size[b, :c, h, 0] = np.where(seen, np.abs(q[b, :c, h]) @ np.abs(k).T, 0).max(1) * scale
    return out, mass, size


class HostDrafts(HostPages):
    """The cache's rules with kv_pages_accept; `rows_moved` lists the moves of its
    last call as ((page, slot) from, to), in order."""

    def accept(self, seqs, counts, max_rows, paths, max_path):
        self.moves, self.rows_moved = [], []
        if not self._listed(seqs):
            return ESEQ
        codes = []
        for s, c, p in zip(seqs, counts, paths):
            if not (0 <= c <= max_rows and c <= self.len[s] and len(p) <= min(c, max_path)):
                codes.append(ELEN)
        if codes:
            return min(codes)
        moved = []
        for s, c, p in zip(seqs, counts, paths):
            first = self.len[s] - c
            if any(not 0 <= r < c for r in p) or any(x >= y for x, y in zip(p, p[1:])):
                codes.append(EPATH)
                # rows before the first that is out of place are looked at all the same
            at = lambda pos: (self.table[s][pos // self.P], pos % self.P)
            before = -1
            for j, r in enumerate(p):
                if r <= before or r >= c:
                    before = r
                    continue
                before = r
                if r != j:
                    moved.append((at(first + r), at(first + j)))
                    if self.refs[at(first + j)[0]] > 1:
                        codes.append(ESHARED)
            end = first + len(p)
            if end < self.len[s] and end % self.P and self.refs[at(end)[0]] > 1:
                codes.append(ESHARED)
        if codes:
            return min(codes)
        self.rows_moved = moved
        keep = [self.len[s] - c + len(p) for s, c, p in zip(seqs, counts, paths)]
        for s, x in zip(seqs, keep):
            for j in range(self.blocks(x), self.max_blocks):
                if self.table[s][j] >= 0:
                    self.refs[self.table[s][j]] -= 1
                    self.table[s][j] = -1
            self.len[s] = x
        return OK
