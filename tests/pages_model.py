"""The paged key/value cache on the host, one page at a time, and attention
over it in 64 bits: what the tests compare the library with."""
import numpy as np

OK, ESEQ, ELEN, ESHARED, EFULL = 0, 1, 2, 3, 4


class HostPages:
    """Tables, references and lengths by the rules of dllm_rps.h; `moves` lists
    the page copies (from, to) of the last call, in order."""

    def __init__(self, n_pages, page_len, max_seqs, max_blocks):
        self.P, self.max_blocks = page_len, max_blocks
        self.refs = [0] * n_pages
        self.table = [[-1] * max_blocks for _ in range(max_seqs)]
        self.len = [0] * max_seqs
        self.moves = []

    def blocks(self, m):
        return -(-m // self.P)

    def _listed(self, seqs):
        return all(0 <= s < len(self.len) for s in seqs) and len(set(seqs)) == len(seqs)

    def _take(self, wants):
        """wants: (sequence, block) in call order."""
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if len(free) < len(wants):
            return False
        for (s, j), p in zip(wants, free):
            self.table[s][j], self.refs[p] = p, 1
        return True

    def grow(self, seqs, add):
        self.moves = []
        if not self._listed(seqs):
            return ESEQ
        if any(a < 0 or self.len[s] + a > self.max_blocks * self.P for s, a in zip(seqs, add)):
            return ELEN
        wants = [(s, j) for s, a in zip(seqs, add) for j in range(self.blocks(self.len[s]), self.blocks(self.len[s] + a))]
        if not self._take(wants):
            return EFULL
        for s, a in zip(seqs, add):
            self.len[s] += a
        return OK

    def fork(self, src, dst, keep=None):
        self.moves = []
        if not self._listed(dst) or any(not 0 <= s < len(self.len) for s in src) or any(self.len[d] for d in dst):
            return ESEQ
        m = [self.len[s] for s in src] if keep is None else list(keep)
        if any(x < 0 or x > self.len[s] for x, s in zip(m, src)):
            return ELEN
        cut = [(d, x // self.P) for d, x in zip(dst, m) if x % self.P]
        if not self._take(cut):
            return EFULL
        for s, d, x in zip(src, dst, m):
            for j in range(x // self.P):
                self.table[d][j] = self.table[s][j]
                self.refs[self.table[s][j]] += 1
            if x % self.P:
                self.moves.append((self.table[s][x // self.P], self.table[d][x // self.P]))
        for d, x in zip(dst, m):
            self.len[d] = x
        return OK

    def free(self, seqs, keep=None):
        self.moves = []
        if not self._listed(seqs):
            return ESEQ
        m = [0] * len(seqs) if keep is None else list(keep)
        if any(x < 0 or x > self.len[s] for x, s in zip(m, seqs)):
            return ELEN
        if any(x < self.len[s] and x % self.P and self.refs[self.table[s][x // self.P]] > 1 for x, s in zip(m, seqs)):
            return ESHARED
        for s, x in zip(seqs, m):
            for j in range(self.blocks(x), self.max_blocks):
                if self.table[s][j] >= 0:
                    self.refs[self.table[s][j]] -= 1
                    self.table[s][j] = -1
            self.len[s] = x
        return OK

    def compact(self):
        used = sum(r > 0 for r in self.refs)
        self.moves = list(zip([p for p in range(used, len(self.refs)) if self.refs[p]],
                              [p for p in range(used) if not self.refs[p]]))
        to = dict(self.moves)
        for a, b in self.moves:
            self.refs[a], self.refs[b] = 0, self.refs[a]
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return used


def attend(q, keys, values, counts, causal, scale):
    """q [n][rows][heads][hd]; keys, values per entry [len][kv heads][hd], all
    float64.  Returns the outputs, sum p |v| per element and the largest
    scale * sum |q| |k| of a row and head (both for error bounds); rows past
    counts[b] are left 0."""
    n, rows, heads, hd = q.shape
    out, mass, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros((n, rows, heads, 1))
    for b in range(n):
        m, c = keys[b].shape[0], counts[b]
        lim = np.array([max(0, min(m, m - c + i + 1)) if causal else m for i in range(c)], dtype=int)
        if m == 0 or c == 0:
            continue
        seen = np.arange(m)[None] < lim[:, None]
        for h in range(heads):
            kv = h // (heads // keys[b].shape[1])
            k, v = keys[b][:, kv], values[b][:, kv]
            z = np.where(seen, q[b, :c, h] @ k.T * scale, -np.inf)
            top = np.where(lim[:, None] > 0, z.max(1, keepdims=True), 0.0)
            w = np.exp(z - top)
            w /= np.maximum(w.sum(1, keepdims=True), 1e-300)
            out[b, :c, h], mass[b, :c, h] = w @ v, w @ np.abs(v)
            size[b, :c, h, 0] = np.where(seen, np.abs(q[b, :c, h]) @ np.abs(k).T, 0).max(1) * scale
    return out, mass, size
