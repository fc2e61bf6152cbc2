"""The paged key/value cache on the GPU against a host model and 64 bits."""
import random

import numpy as np
import pytest
import torch

from tests.pages_model import HostPages, attend, OK, ESEQ, ELEN, ESHARED, EFULL

pytestmark = pytest.mark.gpu
P = pytest.importorskip("paper_2608_11742_amd")

DEV = "cuda:0"


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def new_pages(layers=2, pages=40, heads=2, page=16, hd=64, seqs=12, blocks=9, dtype=torch.bfloat16, seed=0):
    kp = P.KvPages.empty(layers, pages, heads, page, hd, seqs, blocks, dtype=dtype, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(seed)
    kp.k.normal_(generator=g)
    kp.vt.normal_(generator=g)
    return kp


class Both:
    """The library's cache and the host model, held against one another after every call."""

    def __init__(self, **kw):
        self.d = new_pages(**kw)
        self.h = HostPages(self.d.k.shape[1], self.d.page_len, *self.d.table.shape)
        self.k, self.vt = self.d.k.clone(), self.d.vt.clone()
        self.status = ints([99])
        self.check()

    def check(self):
        for a, b in self.h.moves:
            self.k[:, b], self.vt[:, b] = self.k[:, a], self.vt[:, a]
        assert self.d.refs.tolist() == self.h.refs
        assert self.d.table.tolist() == self.h.table
        assert self.d.len.tolist() == self.h.len
        assert torch.equal(self.d.k, self.k) and torch.equal(self.d.vt, self.vt)

    def call(self, name, *lists):
        want = getattr(self.h, name)(*lists)
        if want != OK:
            self.h.moves = []
        t = [None if x is None else ints(list(x)) for x in lists]
        if name == "grow":
            P.kv_pages_grow(self.d, t[0], t[1], self.status)
        elif name == "fork":
            P.kv_pages_fork(self.d, t[0], t[1], self.status, keep=t[2] if len(t) > 2 else None)
        else:
            P.kv_pages_free(self.d, t[0], self.status, keep=t[1] if len(t) > 1 else None)
        assert self.status.item() == want, (name, lists)
        self.check()
        return want

    def compact(self):
        used = ints([-1])
        ws = torch.empty(P.kv_pages_compact_workspace_bytes(self.d), dtype=torch.uint8, device=DEV)
        want = self.h.compact()
        P.kv_pages_compact(self.d, used, ws)
        assert used.item() == want
        self.check()


@pytest.mark.parametrize("seed,kw", [
    (0, {}),
    (1, dict(page=32, hd=128, dtype=torch.float32, pages=23)),
    (2, dict(layers=1, heads=1, pages=1100, seqs=40, blocks=70)),     # more pages than planning threads
    (3, dict(page=256, heads=3, pages=9, blocks=3)),                  # pages of several copy units
    (4, dict(pages=2500, seqs=600, blocks=60, heads=1, layers=1)),    # tables past what one workgroup clears
])
def test_random_calls(seed, kw):
    rng = random.Random(seed)
    both = Both(seed=seed, **kw)
    n_seqs, blocks = both.d.table.shape
    P_ = both.d.page_len
    seen = set()
    for _ in range(60):
        what = rng.choice(["grow", "grow", "fork", "fork", "free", "compact"])
        held = [s for s in range(n_seqs) if both.h.len[s]]
        empty = [s for s in range(n_seqs) if not both.h.len[s]]
        if what == "grow":
            seqs = rng.sample(range(n_seqs), rng.randint(1, n_seqs))
            seen.add((what, both.call("grow", seqs, [rng.choice([0, 1, 5, P_, 2 * P_ + 3]) for _ in seqs])))
        elif what == "fork" and held and empty:
            dst = rng.sample(empty, rng.randint(1, len(empty)))
            src = [rng.choice(held) for _ in dst]
            keep = None if rng.random() < 0.4 else [rng.randint(0, both.h.len[s]) for s in src]
            seen.add((what, both.call("fork", src, dst, keep)))
        elif what == "free" and held:
            seqs = rng.sample(held, rng.randint(1, len(held)))
            keep = None if rng.random() < 0.5 else [rng.randint(0, both.h.len[s]) for s in seqs]
            seen.add((what, both.call("free", seqs, keep)))
        elif what == "compact":
            both.compact()
    assert ("grow", OK) in seen and ("fork", OK) in seen and ("free", OK) in seen


def test_errors_change_nothing():
    both = Both(pages=10, page=16, seqs=6, blocks=5)
    assert both.call("grow", [0, 1], [40, 32]) == OK                  # 3 + 2 pages
    assert both.call("grow", [0, 0], [1, 1]) == ESEQ                  # listed twice
    assert both.call("grow", [2, 6], [1, 1]) == ESEQ
    assert both.call("grow", [-1], [1]) == ESEQ
    assert both.call("grow", [2], [-1]) == ELEN
    assert both.call("grow", [0], [41]) == ELEN                       # past max_blocks
    assert both.call("grow", [0], [2 ** 31 - 1]) == ELEN
    assert both.call("grow", [2, 3, 4], [32, 32, 32]) == EFULL        # 6 of 5
    assert both.call("grow", [3, 2], [80, 0]) == OK                   # exactly the rest
    assert both.call("grow", [2], [1]) == EFULL
    assert both.call("fork", [0], [1]) == ESEQ                        # target in use
    assert both.call("fork", [0], [6]) == ESEQ
    assert both.call("fork", [7], [2]) == ESEQ
    assert both.call("fork", [0, 1], [2, 2]) == ESEQ
    assert both.call("fork", [0], [2], [41]) == ELEN
    assert both.call("fork", [0], [2], [-1]) == ELEN
    assert both.call("fork", [0], [2]) == EFULL                       # the cut page has nowhere to go
    assert both.call("fork", [0, 0], [2, 4], [32, 16]) == OK          # whole pages need none
    assert both.call("free", [0], [20]) == ESHARED                    # page 1 is held by sequence 2 too
    assert both.call("free", [0, 2], [20, 0]) == ESHARED              # references as before the call
    assert both.call("free", [0], [40]) == OK                         # nothing dropped
    assert both.call("free", [0], [35]) == OK                         # inside its own page
    assert both.call("free", [0], [36]) == ELEN
    assert both.call("free", [1, 1]) == ESEQ
    assert both.call("free", [2], [16]) == OK
    assert both.call("free", [0], [20]) == OK                         # held once now
    assert both.call("fork", [5], [5], [0]) == OK             # an empty one of itself
    assert both.call("fork", [5, 0], [5, 2], None) == ESEQ    # 2 is in use


def test_sources_as_before_the_call():
    both = Both(pages=20)
    assert both.call("grow", [0], [20]) == OK
    # 2 is filled from 0 by the same call that reads it: it is read empty
    assert both.call("fork", [0, 2, 0], [2, 3, 4]) == OK
    assert both.h.len[3] == 0


def test_full_and_empty_pool():
    both = Both(pages=8, seqs=4, blocks=8)
    both.compact()                                                    # nothing held
    assert both.call("grow", [1], [8 * 16]) == OK
    both.compact()                                                    # nothing free
    assert both.call("free", [1], [1]) == OK
    both.compact()
    assert both.call("grow", [0, 2], [3 * 16, 64]) == OK
    assert both.call("free", [0]) == OK
    both.compact()


def test_needs_past_31_bits():
    """Tables of the largest length: 32 sequences that ask for 2^26 pages each, 2^31 together."""
    kp = P.KvPages.empty(1, 4, 1, 16, 64, 32, 1 << 26, device=DEV)
    status, seqs = ints([99]), ints(list(range(32)))
    for n in (32, 31, 1):
        P.kv_pages_grow(kp, seqs[:n], ints([1 << 30] * n), status)
        assert status.item() == EFULL
        assert kp.len.tolist() == [0] * 32 and kp.refs.tolist() == [0] * 4
    P.kv_pages_grow(kp, seqs, ints([17] + [0] * 30 + [20]), status)
    assert status.item() == OK
    assert kp.len.tolist() == [17] + [0] * 30 + [20] and kp.refs.tolist() == [1] * 4
    assert kp.table[:, :3].tolist() == [[0, 1, -1]] + [[-1] * 3] * 30 + [[2, 3, -1]]
    P.kv_pages_free(kp, seqs, status)
    assert status.item() == OK and kp.refs.tolist() == [0] * 4 and bool((kp.table[31] == -1).all())


# ---------------------------------------------------------------- rows

def hold(kp, lens, seed=0):
    """Sequences of these lengths on shuffled pages (written through the arrays: the calls have tests of their own)."""
    rng = random.Random(seed)
    ids = rng.sample(range(kp.k.shape[1]), kp.k.shape[1])
    refs, table = torch.zeros(kp.k.shape[1], dtype=torch.int32), torch.full(kp.table.shape, -1, dtype=torch.int32)
    for s, m in enumerate(lens):
        for j in range(-(-m // kp.page_len)):
            table[s, j] = ids.pop()
            refs[table[s, j]] = 1
    kp.refs.copy_(refs)
    kp.table.copy_(table)
    kp.len[:len(lens)] = ints(lens)
    return kp


def gather(kp, layer, s):
    """Keys and values [len][heads][hd] of a sequence, float64 on the host."""
    m, at = int(kp.len[s]), kp.table[s][kp.table[s] >= 0].long()
    k = kp.k[layer][at].double().permute(0, 2, 1, 3).reshape(-1, kp.n_kv_heads, kp.head_dim)[:m]
    v = kp.vt[layer][at].double().permute(0, 3, 1, 2).reshape(-1, kp.n_kv_heads, kp.head_dim)[:m]
    return k.cpu().numpy(), v.cpu().numpy()


def write_reference(kp, layer, seqs, k, v, counts):
    wk, wv = kp.k.clone(), kp.vt.clone()
    for b, s in enumerate(seqs):
        if not 0 <= s < kp.table.shape[0] or s in seqs[b + 1:]:
            continue
        m = int(kp.len[s])
        for i in range(counts[b]):
            pos = m - counts[b] + i
            if pos < 0:
                continue
            page = int(kp.table[s, pos // kp.page_len])
            if int(kp.refs[page]) > 1:
                continue
            wk[layer, page, :, pos % kp.page_len] = k[b, i]
            x = v[b, i].double()
            wv[layer, page, :, :, pos % kp.page_len] = (x.clamp(-65504, 65504) if kp.vt.dtype == torch.float16 else x).to(kp.vt.dtype)
    return wk, wv


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page,hd,heads,rows,lens", [
    (16, 64, 1, 1, [1, 16, 17, 0, 33]),
    (16, 128, 3, 5, [5, 7, 3, 100]),               # the third has fewer positions than rows
    (32, 64, 2, 64, [64, 70, 127]),
    (64, 128, 2, 97, [97, 130, 513, 160]),
    (256, 64, 1, 200, [200, 456]),
    (128, 128, 1, 130, [131]),
])
def test_write(dtype, page, hd, heads, rows, lens):
    kp = hold(new_pages(pages=2 + sum(-(-m // page) for m in lens), heads=heads, page=page, hd=hd, seqs=len(lens) + 1,
                        blocks=max(1, -(-max(lens) // page)), dtype=dtype), lens)
    n = len(lens)
    g = torch.Generator(device=DEV).manual_seed(1)
    qkv = torch.empty(n, rows, 3 * heads, hd, dtype=dtype, device=DEV).normal_(generator=g)
    k, v = qkv[:, :, heads:2 * heads], qkv[:, :, 2 * heads:]
    v[0, 0, 0, 0] = 1e6 if dtype == torch.bfloat16 else 1.0           # past binary16
    seqs = list(range(n))[::-1]
    for counts in ([rows] * n, [rows - i * rows // n for i in range(n)]):
        wk, wv = write_reference(kp, 1, seqs, k, v, counts)
        P.kv_pages_write(kp, 1, ints(seqs), k, v, n_rows=None if counts == [rows] * n else ints(counts))
        assert torch.equal(kp.k, wk) and torch.equal(kp.vt, wv)


def test_write_leaves_what_is_not_its_own():
    kp = hold(new_pages(seqs=6), [40, 37, 20, 16])
    kp.refs[kp.table[1, 1].long()] = 2                                # positions 16..31 of sequence 1 held twice
    g = torch.Generator(device=DEV).manual_seed(1)
    k = torch.empty(6, 30, 2, 64, dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    v = torch.empty(2, 6, 30, 64, dtype=torch.bfloat16, device=DEV).normal_(generator=g).permute(1, 2, 0, 3)
    seqs, counts = [0, 1, 0, -1, 6, 2], [30, 25, 9, 30, 30, 0]        # 0 twice: the last entry's 9 rows alone
    wk, wv = write_reference(kp, 0, seqs, k, v, counts)
    P.kv_pages_write(kp, 0, ints(seqs), k, v, n_rows=ints(counts))
    assert torch.equal(kp.k, wk) and torch.equal(kp.vt, wv)
    counts = [-5, 99, -1, 0, 0, 99]                                   # clamped to 0 .. 30
    wk, wv = write_reference(kp, 0, seqs, k, v, [0, 30, 0, 0, 0, 30])
    P.kv_pages_write(kp, 0, ints(seqs), k, v, n_rows=ints(counts))
    assert torch.equal(kp.k, wk) and torch.equal(kp.vt, wv)


# ---------------------------------------------------------------- attention

def poison(kp):
    """NaN wherever no sequence has a position, the rest of last pages too."""
    live = torch.zeros(kp.k.shape[1], kp.page_len, dtype=torch.bool)
    for s, m in enumerate(kp.len.tolist()):
        for j in range(-(-m // kp.page_len)):
            live[int(kp.table[s, j]), :min(kp.page_len, m - j * kp.page_len)] = True
    live = live.to(DEV)
    kp.k.masked_fill_(~live[None, :, None, :, None], float("nan"))
    kp.vt.masked_fill_(~live[None, :, None, None, :], float("nan"))


def check_attention(kp, layer, seqs, q, counts, causal=False, scale=None, keys=None, **kw):
    n, rows, heads, hd = q.shape
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    ws = torch.full((P.kv_pages_attention_workspace_bytes(kp, n, rows, heads),), 255, dtype=torch.uint8, device=DEV)
    P.kv_pages_attention(kp, layer, ints(seqs), q, out, ws, n_rows=None if counts is None else ints(counts),
                         causal=causal, scale=scale, **kw)
    counts = [rows] * n if counts is None else [min(max(c, 0), rows) for c in counts]
    none = np.zeros((0, kp.n_kv_heads, hd))
    kv = keys or [gather(kp, layer, s) if 0 <= s < kp.table.shape[0] else (none, none) for s in seqs]
    want, mass, size = attend(q.double().cpu().numpy(), [k for k, _ in kv], [v for _, v in kv], counts, causal,
                              hd ** -0.5 if scale is None else scale)
    got = out.double().cpu().numpy()
    longest = max(k.shape[0] for k, _ in kv)
    # a score's error is at most (hd + 4) roundings of its sum of products: a
    # relative error of twice that in every weight; the sums over the keys add
    # one rounding a key; all relative to sum p |v|
    tol = mass * 2.0 ** -24 * (2 * (hd + 4) * size + longest + 64)
    if q.dtype == torch.bfloat16:
        # weights rounded to binary16 (half a step, 2^-11), the output to bf16 (2^-8)
        tol += mass * 2.0 ** -11 + np.abs(want) * 2.0 ** -8
    for b, c in enumerate(counts):
        assert np.all(got[b, c:] == 7.0)                              # rows past the count as they were
        diff, t = np.abs(got[b, :c] - want[b, :c]), tol[b, :c] + 1e-30
        assert np.all(diff <= t), (b, float(np.max(diff / t)))
    return out


def queries(n, rows, heads, hd, dtype, seed=5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(n, rows, heads + 2, hd, dtype=dtype, device=DEV).normal_(generator=g)[:, :, :heads]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,hd,page,heads,kv,rows,lens", [
    (torch.bfloat16, 64, 16, 1, 1, 1, [1]),
    (torch.bfloat16, 128, 64, 4, 4, 1, [1, 63, 64, 65, 200]),
    (torch.bfloat16, 64, 16, 8, 2, 1, [0, 5, 300, 1000]),             # an empty sequence
    (torch.bfloat16, 128, 128, 8, 1, 3, [2, 400, 129]),               # fewer positions than causal rows
    (torch.bfloat16, 128, 32, 2, 2, 33, [33, 60, 500]),
    (torch.bfloat16, 64, 256, 2, 1, 65, [300, 1]),
    (torch.bfloat16, 128, 16, 2, 2, 130, [130, 260]),
    (torch.bfloat16, 64, 32, 6, 2, 50, [700, 50, 51]),
    (torch.float32, 64, 16, 2, 2, 1, [1, 40, 500]),
    (torch.float32, 128, 32, 4, 2, 17, [17, 200]),
    (torch.float32, 64, 64, 3, 3, 70, [70, 333, 0]),
    (torch.float32, 128, 256, 1, 1, 150, [400]),
])
def test_attention(dtype, hd, page, heads, kv, rows, lens, causal):
    kp = hold(new_pages(pages=2 + sum(-(-m // page) for m in lens), heads=kv, page=page, hd=hd, seqs=len(lens),
                        blocks=max(1, -(-max(lens) // page)), dtype=dtype), lens)
    poison(kp)
    n = len(lens)
    seqs = list(range(n))[::-1]
    q = queries(n, rows, heads, hd, dtype)
    check_attention(kp, 1, seqs, q, None, causal, max_len=max(lens))
    check_attention(kp, 1, seqs, q, [max(0, rows - 2 * i) for i in range(n)], causal)


def shared_batch(dtype, hd, page, kv, prefix, lens, seed=0):
    """Sequence 0 holds the prefix; 1 .. n share its whole pages and go on alone."""
    whole = prefix // page
    extra = [m - min(m, whole * page) for m in lens]
    total = -(-prefix // page) + sum(-(-x // page) + 1 for x in extra)
    kp = new_pages(pages=total + 2, heads=kv, page=page, hd=hd, seqs=len(lens) + 2,
                   blocks=max(-(-max(lens + [prefix]) // page), 1), dtype=dtype, seed=seed)
    hold(kp, [prefix], seed)
    free = [p for p in range(total + 2) if int(kp.refs[p]) == 0]
    random.Random(seed).shuffle(free)
    table, refs = kp.table.cpu(), kp.refs.cpu()
    for i, m in enumerate(lens, 1):
        for j in range(-(-m // page)):
            table[i, j] = table[0, j] if j < whole else free.pop()
            refs[table[i, j]] += 1
    kp.table.copy_(table)
    kp.refs.copy_(refs)
    kp.len[1:1 + len(lens)] = ints(lens)
    return kp


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype,hd,page,heads,kv,rows,prefix,lens", [
    (torch.bfloat16, 128, 64, 4, 4, 32, 512, [544] * 5),              # a lookahead's branches
    (torch.bfloat16, 128, 64, 2, 2, 32, 531, [532, 600, 563]),        # the prefix ends inside a page
    (torch.bfloat16, 64, 16, 8, 2, 1, 700, [701, 900, 705, 716, 1300]),
    (torch.bfloat16, 64, 32, 2, 2, 7, 96, [100, 20, 0, 97]),          # sequences shorter than the prefix
    (torch.bfloat16, 128, 16, 4, 1, 40, 15, [60, 61]),                # no whole page is shared
    (torch.bfloat16, 64, 128, 2, 2, 3, 1024, [1024, 1024]),           # nothing behind the prefix
    (torch.float32, 64, 16, 2, 2, 19, 203, [204, 260, 333]),
    (torch.float32, 128, 64, 4, 2, 1, 1000, [1001, 1040] * 9),
])
def test_attention_over_a_shared_prefix(dtype, hd, page, heads, kv, rows, prefix, lens, causal):
    kp = shared_batch(dtype, hd, page, kv, prefix, lens)
    poison(kp)
    n = len(lens)
    seqs = list(range(1, n + 1))
    q = queries(n, rows, heads, hd, dtype)
    kw = dict(prefix_seq=0, max_len=max(lens))
    check_attention(kp, 0, seqs, q, None, causal, shared_len=prefix, **kw)
    # a prefix given too long ends where its sequence does; a shorter one, and a wrong max_len, change nothing but time
    check_attention(kp, 0, seqs, q, [rows - i % 2 * (rows // 2) for i in range(n)], causal, shared_len=prefix + 1000, **kw)
    check_attention(kp, 0, seqs, q, None, causal, shared_len=max(1, prefix // 2), prefix_seq=0, max_len=1)
    # entries that are no sequence, twice the same one, and the prefix itself
    check_attention(kp, 0, [-1, 1, 1, 99, 0][:max(n, 2)], queries(min(5, max(n, 2)), rows, heads, hd, dtype), None,
                    causal, shared_len=prefix, **kw)


@pytest.mark.parametrize("hd,page,n,rows,prefix,lens,counts", [
    (64, 64, 12, 32, 192, [224], None),                               # whole steps, equal branches
    (128, 16, 13, 25, 173, [198, 160, 0, 339], None),                 # an odd count of blocks, one ends inside the prefix
    (64, 128, 7, 61, 256, [317, 280, 600], [61, 0, 17]),              # two blocks an entry, nothing behind the prefix's pages in some
    (128, 32, 12, 24, 31, [55, 31, 90], [24, 5, 23]),                 # no whole page is shared
])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_of_many_branches(hd, page, n, rows, prefix, lens, counts, causal):
    """Enough blocks of rows to fill the chip: 32 heads, entries of about whole blocks."""
    lens = [lens[i % len(lens)] for i in range(n)]
    kp = shared_batch(torch.bfloat16, hd, page, 32, prefix, lens)
    poison(kp)
    q = queries(n, rows, 32, hd, torch.bfloat16)
    check_attention(kp, 1, list(range(1, n + 1)), q, None if counts is None else [counts[i % len(counts)] for i in range(n)],
                    causal, prefix_seq=0, shared_len=prefix, max_len=max(lens))


@pytest.mark.parametrize("hd,page,heads,kv,n,rows,prefix,lens", [
    (128, 16, 2, 2, 5, 130, 173, [303, 180, 90, 0, 500]),             # entries by themselves fill workgroups
    (64, 32, 4, 4, 3, 70, 1000, [1070, 1100, 900]),                   # and are divided
    (128, 16, 8, 8, 20, 33, 117, [150, 117, 160]),
    (64, 64, 4, 4, 4, 128, 700, [828, 1500, 60]),
    (128, 64, 8, 2, 6, 40, 130, [170, 300, 131]),                     # grouped heads
    (64, 128, 32, 32, 7, 60, 640, [700, 655, 641, 100]),              # two blocks an entry, in pairs
    (128, 32, 32, 32, 9, 17, 517, [534, 520, 0, 612]),                # blocks half empty
    (64, 16, 32, 4, 9, 5, 530, [535, 530, 700]),                      # rows of grouped heads in a block
])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_of_entries_and_parts(hd, page, heads, kv, n, rows, prefix, lens, causal):
    """Batches about where one way to take them over a prefix gives place to another."""
    lens = [lens[i % len(lens)] for i in range(n)]
    kp = shared_batch(torch.bfloat16, hd, page, kv, prefix, lens)
    poison(kp)
    q = queries(n, rows, heads, hd, torch.bfloat16)
    counts = [max(0, rows - 7 * (i % 4)) for i in range(n)]
    for most in (max(lens), 1, 20000):
        check_attention(kp, 1, list(range(1, n + 1)), q, counts, causal, prefix_seq=0, shared_len=prefix, max_len=most)


@pytest.mark.parametrize("hd,page,heads,kv,n,rows,prefix,lens,causal", [
    (64, 64, 32, 32, 3, 50, 16400, [16450, 16433, 16600], False),     # stacked rows end inside a row tile
    (128, 128, 64, 8, 5, 26, 16500, [16526, 16700, 16550, 16390, 0], True),   # grouped heads, one entry inside the prefix, one empty
    (64, 256, 16, 4, 1, 300, 0, [65800], True),                       # one sequence, nothing shared
])
def test_attention_of_heavy_batches(hd, page, heads, kv, n, rows, prefix, lens, causal):
    """Many rows over many keys, in ranges that are joined."""
    kp = shared_batch(torch.bfloat16, hd, page, kv, prefix, lens) if prefix else hold(
        new_pages(pages=lens[0] // page + 3, heads=kv, page=page, hd=hd, seqs=1, blocks=-(-lens[0] // page)), lens)
    poison(kp)
    q = queries(n, rows, heads, hd, torch.bfloat16)
    check_attention(kp, 0, list(range(1, n + 1)) if prefix else [0], q, [rows, 3, rows - 1, rows, 1][:n], causal, prefix_seq=0,
                    shared_len=prefix, max_len=max(lens))


def test_attention_extremes():
    """Scores far apart, infinities among the values, keys that are not numbers in one sequence alone."""
    kp = hold(new_pages(seqs=4, pages=60, blocks=20), [300, 200, 290, 17])
    q = queries(4, 9, 2, 64, torch.bfloat16)
    kp.k.mul_(20)                                                     # scores up to some hundreds
    check_attention(kp, 0, [0, 1, 2, 3], q, None)
    check_attention(kp, 0, [0, 1, 2, 3], q, None, scale=1e-3)
    clean = check_attention(kp, 0, [0, 1, 2, 3], q, None, causal=True)
    kp.k[0, kp.table[1, 0].long()] = float("nan")
    out = torch.zeros_like(q)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, 4, 9, 2), dtype=torch.uint8, device=DEV)
    P.kv_pages_attention(kp, 0, ints([0, 1, 2, 3]), q, out, ws, causal=True)
    assert torch.equal(out[[0, 2, 3]], clean[[0, 2, 3]]) and out[1].isnan().all()


@pytest.mark.parametrize("n,rows,keys,shared", [
    (1024, 1, 1500, 0),          # rows of single tokens
    (1, 65536, 20000, 0),        # many rows
    (400, 32, 8000, 8000),       # branches over a prefix
    (2, 16, 60000, 60000),       # ranges joined
])
def test_attention_weights_far_below_the_largest(n, rows, keys, shared):
    """Key 0 outweighs every other one by 2^25, its value is 0 and theirs 1: the
    output is what the others weigh together, a bf16 rounding (2^-8) and their
    weights' rounding (2^-17 of binary16 with 2^8 the largest: half a step of
    2^-24 is 2^-8 of it) away."""
    page, hd = 64, 64
    whole = -(-keys // page)
    kp = P.KvPages.empty(1, whole, 1, page, hd, 1024, whole, device=DEV)
    kp.k.zero_()
    kp.vt.fill_(1)
    kp.k[0, 0, 0, 0, 0] = 4.34375
    kp.vt[0, 0, 0, :, 0] = 0
    kp.table[:] = torch.arange(whole, dtype=torch.int32, device=DEV)
    kp.len.fill_(keys)
    kp.refs.fill_(1024)
    q = torch.zeros(n, rows, 1, hd, dtype=torch.bfloat16, device=DEV)
    q[..., 0] = 4
    out = torch.empty_like(q)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, n, rows, 1), dtype=torch.uint8, device=DEV)
    P.kv_pages_attention(kp, 0, ints(list(range(n))), q, out, ws, shared_len=shared, max_len=keys, scale=1.0)
    want = (keys - 1) / (np.exp(4 * 4.34375) + keys - 1)
    diff = (out.double() / want - 1).abs().max().item()
    assert diff <= 2.0 ** -8 + 2.0 ** -7.9 + 2.0 ** -10


def test_attention_strides_and_heads_first():
    kp = hold(new_pages(seqs=3, pages=60, blocks=20, heads=4), [300, 64, 290])
    g = torch.Generator(device=DEV).manual_seed(3)
    q = torch.empty(3, 8, 11, 64, dtype=torch.bfloat16, device=DEV).normal_(generator=g).permute(0, 2, 1, 3)
    want = check_attention(kp, 1, [0, 1, 2], q, None)
    buf = torch.zeros(3, 8, 15, 80, dtype=torch.bfloat16, device=DEV)
    out = buf[:, :, 2:13, 8:72].permute(0, 2, 1, 3)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, 3, 11, 8), dtype=torch.uint8, device=DEV)
    P.kv_pages_attention(kp, 1, ints([0, 1, 2]), q, out, ws)
    assert torch.equal(out, want)
    buf[:, :, 2:13, 8:72] = 0
    assert not buf.any()
    one = q[1:2, :1].expand(3, 11, 8, 64)                             # the same row everywhere
    check_attention(kp, 1, [0, 1, 2], one, None)


# ---------------------------------------------------------------- together

def round_of(kp, st, roots, branches, block, k, v, q, out, ws, shared):
    P.kv_pages_free(kp, branches, st[0:1])
    P.kv_pages_fork(kp, roots, branches, st[1:2])
    P.kv_pages_grow(kp, branches, block, st[2:3])
    for layer in range(kp.k.shape[0]):
        P.kv_pages_write(kp, layer, branches, k, v)
        P.kv_pages_attention(kp, layer, branches, q, out[layer], ws, prefix_seq=0, shared_len=shared)


def test_rounds_of_a_search_captured_and_replayed():
    """Fork, grow, write and attend in one graph, replayed between eager calls
    on another stream; every replay against the tables and 64 bits."""
    kp = new_pages(pages=60, seqs=8, blocks=8, layers=2)
    st = ints([9, 9, 9])
    P.kv_pages_grow(kp, ints([0]), ints([75]), st[0:1])
    n, rows = 5, 20
    roots, branches, block = ints([0] * n), ints(list(range(1, 1 + n))), ints([rows] * n)
    g = torch.Generator(device=DEV).manual_seed(3)
    k, v, q = (torch.empty(n, rows, 2, 64, dtype=torch.bfloat16, device=DEV).normal_(generator=g) for _ in range(3))
    out = torch.zeros(2, n, rows, 2, 64, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, n, rows, 2), dtype=torch.uint8, device=DEV)
    args = (kp, st, roots, branches, block, k, v, q, out, ws, 75)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        round_of(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_of(*args)
    for replay in range(3):
        for t in (k, v, q):
            t.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        assert st.tolist() == [0, 0, 0] and kp.len.tolist() == [75] + [95] * n + [0, 0]
        got = out.clone()
        for layer in range(2):
            kv = [gather(kp, layer, s) for s in range(1, 1 + n)]
            for b in range(n):
                assert np.array_equal(kv[b][0][75:], k[b].double().cpu().numpy())
                assert np.array_equal(kv[b][1][75:], v[b].half().double().cpu().numpy())
            assert torch.equal(check_attention(kp, layer, list(range(1, 1 + n)), q, None, keys=kv, shared_len=75), got[layer])
        with torch.cuda.stream(side):
            round_of(*args)                                           # the same round again, eager
        torch.cuda.synchronize()
        assert torch.equal(out, got)


def test_refusals():
    kp = hold(new_pages(seqs=3), [40, 20, 0])
    q = queries(2, 3, 2, 64, torch.bfloat16).contiguous()
    out, ws = torch.empty_like(q), torch.empty(P.kv_pages_attention_workspace_bytes(kp, 2, 3, 2), dtype=torch.uint8, device=DEV)
    two, st = ints([0, 1]), ints([0])
    bad = [
        lambda: P.kv_pages_attention(kp, 0, two.long(), q, out, ws),
        lambda: P.kv_pages_attention(kp, 0, ints([0]), q, out, ws),
        lambda: P.kv_pages_attention(kp, 0, two, q.float(), out, ws),
        lambda: P.kv_pages_attention(kp, 0, two, q.transpose(2, 3).contiguous().transpose(2, 3), out, ws),
        lambda: P.kv_pages_attention(kp, 0, two, q, out[:, :2], ws),
        lambda: P.kv_pages_attention(kp, 0, two, q, out, ws, n_rows=ints([1])),
        lambda: P.kv_pages_attention(kp, 0, two, q[..., :32], out[..., :32], ws),
        lambda: P.kv_pages_write(kp, 0, two, q, q[:, :2]),
        lambda: P.kv_pages_write(kp, 0, two, q[:, :, :1], q[:, :, :1]),
        lambda: P.kv_pages_grow(kp, two, ints([1]), st),
        lambda: P.kv_pages_grow(kp, two.cpu(), two, st),
        lambda: P.kv_pages_fork(kp, two, ints([2]), st),
        lambda: P.kv_pages_free(kp, two, ints([0, 0])),
        lambda: P.KvPages(kp.k, kp.vt.float(), kp.refs, kp.table, kp.len),
        lambda: P.KvPages(kp.k, kp.vt, kp.refs[:-1], kp.table, kp.len),
        lambda: P.KvPages(kp.k, kp.vt, kp.refs, kp.table, kp.len.cpu()),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    refused = [
        lambda: P.kv_pages_attention(kp, 2, two, q, out, ws),
        lambda: P.kv_pages_attention(kp, 0, two, q, out, ws, shared_len=-1),
        lambda: P.kv_pages_attention(kp, 0, two, q, out, ws, prefix_seq=3, shared_len=16),
        lambda: P.kv_pages_attention(kp, 0, two, q, out, ws, scale=0.0),
        lambda: P.kv_pages_attention(kp, 0, two, q, out[:, :1].expand(2, 3, 2, 64), ws),
        lambda: P.kv_pages_attention(kp, 0, two, q, out, ws[1:]),
        lambda: P.kv_pages_write(kp, -1, two, q, q),
        lambda: P.kv_pages_compact(kp, st, ws[:16]),
    ]
    before = (kp.k.clone(), kp.vt.clone(), kp.refs.clone(), kp.table.clone(), kp.len.clone())
    for call in refused:
        with pytest.raises(P.binding.DllmError):
            call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, (kp.k, kp.vt, kp.refs, kp.table, kp.len)))
