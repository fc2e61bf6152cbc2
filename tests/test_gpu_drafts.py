"""Rotations, appended rows, drafted trees and their acceptance on the GPU,
against a host model and 64 bits."""
import random

import numpy as np
import pytest
import torch

from tests.drafts_model import EPATH, HostDrafts, attend_tree, frequencies, rotate, sees, words
from tests.pages_model import OK, ESEQ, ELEN, ESHARED
from tests.pages_ways import WAYS, division
from tests.test_gpu_pages import Both, gather, hold, ints, new_pages, poison, queries, shared_batch, write_reference
from tests.test_gpu_pages_ways import TYPES, batch

pytestmark = pytest.mark.gpu
P = pytest.importorskip("paper_2608_11742_amd")

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def normal(*shape, dtype=BF16, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(*shape, dtype=dtype, device=DEV).normal_(generator=g)


def host(x):
    return x.double().cpu().numpy()


# ---------------------------------------------------------------- rotations

def new_rotary(hd, dim=None, layout="halves", norm=False, gains=True, **kw):
    q_gain, k_gain = ((1 + 0.3 * normal(hd, dtype=F32, seed=s) for s in (8, 9)) if norm and gains else (None, None))
    rot = P.Rotary(hd, dim=dim, layout=layout, norm=norm, q_gain=q_gain, k_gain=k_gain, device=DEV, **kw)
    rot.want = dict(dim=rot.dim, pairs=layout == "pairs", norm=norm, eps=kw.get("eps", 1e-5))
    rot.freq_kw = {k: v for k, v in kw.items() if k not in ("eps", "amplitude", "freq")}
    return rot


def turned(rot, x, pos, gain):
    """What x [..., heads, hd] at pos becomes, and how far off it may be.

    Norm: hd products and sums and the root, each off by 2^-24 of the result.
    Angle: the product with the position in 64 bits, rounded at 2^-52 of the
    angle twice, the rest below half a quarter turn rounded to 2^-26 of one; sine
    and cosine 2 units of 2^-23, their factor 2^-24; two products and a sum of
    2^-24 each: 10 units of 2^-24 of both elements of the pair.  bf16 at last."""
    freq, amplitude = frequencies(rot.dim, **rot.freq_kw)
    want, mass = rotate(host(x), pos, freq, amplitude=rot.amplitude, gain=None if gain is None else host(gain), **rot.want)
    unit = 10 + (x.shape[-1] / 2 + 8 if rot.want["norm"] else 0)
    far = np.abs(np.asarray(pos, dtype=np.float64))[..., None, None] * 2.0 ** -51
    tol = mass * (unit * 2.0 ** -24 + far) + 1e-30
    if x.dtype == BF16:
        tol += np.abs(want) * 2.0 ** -8
    return want, tol


def check_turned(got, rot, x, pos, gain):
    want, tol = turned(rot, x, pos, gain)
    diff = np.abs(host(got) - want)
    assert np.all(diff <= tol), float(np.max(diff / tol))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd,dim,layout,norm,n,rows,heads,kv,first,kw", [
    (64, 64, "halves", False, 1, 1, 1, 1, 0, {}),
    (128, 128, "halves", True, 3, 5, 32, 8, 1000, {}),
    (64, 32, "pairs", True, 2, 7, 16, 16, 90, {}),
    (128, 48, "pairs", False, 2, 3, 5, 3, 7, {}),                     # heads that leave a step part empty
    (128, 16, "halves", True, 1, 9, 3, 1, 100000, dict(scaling="ramp", factor=16.0)),
    (64, 48, "halves", False, 5, 2, 9, 2, 1 << 20, dict(scaling="linear", factor=4.0, base=500000.0)),
    (64, 64, "pairs", True, 1, 300, 4, 4, 50, dict(scaling="base", factor=8.0)),
    (128, 0, "halves", True, 2, 4, 4, 2, 3, {}),                      # a norm alone
    (64, 64, "halves", True, 70, 64, 2, 1, 0, dict(eps=0.5)),         # rows fill the chip
    (128, 128, "halves", False, 2, 3, 4, 4, (1 << 31) - 8, {}),       # the last positions there are
    (64, 64, "pairs", False, 2, 3, 4, 4, -1000, {}),
])
def test_rotary(dtype, hd, dim, layout, norm, n, rows, heads, kv, first, kw):
    rot = new_rotary(hd, dim, layout, norm, **kw)
    qkv = normal(n, rows, heads + 2 * kv, hd, dtype=dtype)
    q, k = qkv[:, :, :heads], qkv[:, :, heads:heads + kv]
    rng = random.Random(3)
    pos = [[min(first + rng.randint(0, 5 + i), (1 << 31) - 1) for i in range(rows)] for _ in range(n)]
    qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
    P.rotary_rows(rot, q, qo, k, ko, pos=ints(pos))
    check_turned(qo, rot, q, pos, rot.q_gain)
    check_turned(ko, rot, k, pos, rot.k_gain)
    # one at a time, from an offset, in place
    at = [[first + i for i in range(rows)]] * n
    if first + rows < 1 << 31:
        only = torch.full_like(k, 7)
        P.rotary_rows(rot, None, None, k, only, pos_offset=first)
        check_turned(only, rot, k, at, rot.k_gain)
    before = qkv.clone()
    P.rotary_rows(rot, q, q, pos=ints(pos))
    assert torch.equal(q, qo) and torch.equal(qkv[:, :, heads:], before[:, :, heads:])


def test_rotary_of_ragged_rows_and_strides():
    rot = new_rotary(64, 32, norm=True, gains=False)
    x = normal(3, 8, 5, 64).permute(0, 2, 1, 3)                       # [3, 5, 8, 64], heads outermost
    buf = torch.full((3, 5, 10, 80), 7, dtype=BF16, device=DEV)
    out = buf[:, :, 1:9, 8:72]
    pos = [[10 * b + i for i in range(5)] for b in range(3)]
    P.rotary_rows(rot, x, out, pos=ints(pos), n_rows=ints([5, 0, -3]))
    check_turned(out[0], rot, x[0], pos[0], None)
    assert bool((out[1:] == 7).all())
    P.rotary_rows(rot, x, out, pos=ints(pos), n_rows=ints([2, 99, 1]))
    check_turned(out[1], rot, x[1], pos[1], None)
    assert bool((out[2, 1:] == 7).all())
    out.fill_(7)
    assert bool((buf == 7).all())
    one = x[:1, :1].expand(3, 5, 8, 64)                               # the same row everywhere
    P.rotary_rows(rot, one, out, pos=ints(pos))
    check_turned(out, rot, one, pos, None)


def test_rotary_values():
    """Zeros, infinities and numbers that are none stay in their pair, and in their head under a norm; frequencies and a factor given."""
    for norm in (False, True):
        rot = P.Rotary(64, freq=torch.linspace(0, 1, 32, dtype=torch.float64), amplitude=0.5, norm=norm, layout="pairs", device=DEV)
        x = normal(1, 4, 3, 64, dtype=F32)
        x[0, 0, 0] = 0
        x[0, 1, 1, 5] = float("nan")
        x[0, 2, 2, 40] = float("inf")
        out = torch.empty_like(x)
        P.rotary_rows(rot, x, out, pos_offset=3)
        bad = ~out.isfinite()
        want = torch.zeros_like(bad)
        if norm:
            want[0, 1, 1] = True
            want[0, 2, 2, 40:42] = True                               # inf / inf; the others inf times 0 are 0
        else:
            want[0, 1, 1, 4:6] = want[0, 2, 2, 40:42] = True
        assert torch.equal(bad, want)
        assert not out[0, 0, 0].any()
        rot.want, rot.freq_kw = dict(dim=64, pairs=True, norm=norm, eps=1e-5), {}
        y, _ = rotate(host(x[0, 3]), 6, np.linspace(0, 1, 32), 64, True, 0.5, norm)
        # units as in turned(), a pair is made of two elements of at most 5
        assert np.abs(host(out[0, 3]) - y).max() <= 10 * (10 + 40) * 2.0 ** -24


# ---------------------------------------------------------------- append

def check_append(kp, layer, seqs, q, k, v, counts, rot, pos=None):
    n, rows = k.shape[:2]
    given, counts = counts, [min(max(c, 0), rows) for c in counts]
    k0 = kp.k.clone()
    at = pos if pos is not None else [[(int(kp.len[s]) if 0 <= s < kp.len.shape[0] else 0) - c + i for i in range(rows)]
                                      for s, c in zip(seqs, counts)]
    # the pages with rows turned in 64 bits, and with how far off each may be
    want, tol = turned(rot, k, at, rot.k_gain)
    wk, wv = write_reference(Cast(kp, torch.float64), layer, seqs, torch.from_numpy(want).to(DEV), v, counts)
    tk, _ = write_reference(Cast(kp, torch.float64, 0.0), layer, seqs, torch.from_numpy(tol).to(DEV), v, counts)
    qo = torch.full_like(q, 7)
    P.kv_pages_append(kp, layer, ints(seqs), k, v, rot, q=q, q_out=qo, pos=None if pos is None else ints(pos),
                      n_rows=None if given == [rows] * n else ints(given))
    assert bool(((kp.k.double() - wk).abs() <= tk).all())            # others have no room to differ
    assert torch.equal(kp.vt, wv)
    live = [0 <= s < kp.len.shape[0] for s in seqs]
    for b, c in enumerate(counts):
        c = c if live[b] else 0
        if c:
            check_turned(qo[b, :c], rot, q[b, :c], at[b][:c], rot.q_gain)
        assert bool((qo[b, c:] == 7).all())
    # and without queries
    kp2k = kp.k.clone()
    kp.k.copy_(k0)
    P.kv_pages_append(kp, layer, ints(seqs), k, v, rot, pos=None if pos is None else ints(pos), n_rows=ints(given))
    assert torch.equal(kp.k, kp2k)


class Cast:
    """A cache's keys in another type (or all one value), for write_reference."""

    def __init__(self, kp, dtype, fill=None):
        self.k = kp.k.to(dtype) if fill is None else torch.full(kp.k.shape, fill, dtype=dtype, device=DEV)
        self.vt, self.refs, self.table, self.len, self.page_len = kp.vt, kp.refs, kp.table, kp.len, kp.page_len


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,hd,heads,kv,rows,lens,dim,layout,norm", [
    (16, 64, 1, 1, 1, [1, 16, 17, 0, 33], 64, "halves", False),
    (16, 128, 6, 3, 5, [5, 7, 3, 100], 64, "pairs", True),           # the third has fewer positions than rows
    (32, 64, 2, 2, 64, [64, 70, 127], 16, "halves", True),
    (64, 128, 8, 2, 97, [97, 130, 513, 160], 128, "halves", True),
    (256, 64, 4, 1, 200, [200, 456], 48, "pairs", False),
    (128, 128, 1, 1, 130, [131], 0, "halves", True),
])
def test_append(dtype, page, hd, heads, kv, rows, lens, dim, layout, norm):
    kp = hold(new_pages(pages=2 + sum(-(-m // page) for m in lens), heads=kv, page=page, hd=hd, seqs=len(lens) + 1,
                        blocks=max(1, -(-max(lens) // page)), dtype=dtype), lens)
    n = len(lens)
    rot = new_rotary(hd, dim, layout, norm)
    qkv = normal(n, rows, heads + 2 * kv, hd, dtype=dtype)
    q, k, v = qkv[:, :, :heads], qkv[:, :, heads:heads + kv], qkv[:, :, heads + kv:]
    v[0, 0, 0, 0] = 1e6 if dtype == BF16 else 1.0                     # past binary16
    seqs = list(range(n))[::-1]
    check_append(kp, 1, seqs, q, k, v, [rows] * n, rot)
    pos = [[3000 + 7 * b + i // 2 for i in range(rows)] for b in range(n)]
    check_append(kp, 0, seqs, q, k, v, [rows - i * rows // n for i in range(n)], rot, pos)


def test_append_leaves_what_is_not_its_own():
    kp = hold(new_pages(seqs=6), [40, 37, 20, 16])
    kp.refs[kp.table[1, 1].long()] = 2                                # positions 16..31 of sequence 1 held twice
    rot = new_rotary(64, norm=True)
    q, k, v = normal(6, 30, 4, 64), normal(6, 30, 2, 64, seed=2), normal(2, 6, 30, 64, seed=3).permute(1, 2, 0, 3)
    seqs = [0, 1, 0, -1, 6, 2]                                        # 0 twice: the last entry's 9 rows alone
    for counts in ([30, 25, 9, 30, 30, 0], [-5, 99, -1, 0, 0, 99]):
        check_append(kp, 0, seqs, q, k, v, counts, rot)


def test_append_in_place_and_from_one_row():
    """Queries turned where they are; the same key row for every position."""
    kp = hold(new_pages(seqs=2, heads=2), [70, 33])
    rot = new_rotary(64)
    q = normal(2, 20, 4, 64)
    was = q.clone()
    k, v = normal(1, 1, 2, 64).expand(2, 20, 2, 64), normal(2, 20, 2, 64, seed=4)
    P.kv_pages_append(kp, 0, ints([0, 1]), k, v, rot, q=q, q_out=q)
    for b, m in enumerate((70, 33)):
        at = list(range(m - 20, m))
        check_turned(q[b], rot, was[b], at, None)
        keys, values = gather(kp, 0, b)
        want, tol = turned(rot, k[b], at, None)
        assert np.all(np.abs(keys[m - 20:] - want) <= tol) and np.array_equal(values[m - 20:], host(v[b].half()))


# ---------------------------------------------------------------- trees

def random_tree(rng, rows, wild=False):
    p = [-1 if i == 0 or rng.random() < 0.1 else rng.randint(max(0, i - 1 - rng.randint(0, i)), i - 1) for i in range(rows)]
    if wild:
        p = [rng.choice([x, i, i + 1, 1 << 30, -7, -(1 << 31)]) if rng.random() < 0.3 else x for i, x in enumerate(p)]
    return p


@pytest.mark.parametrize("n,rows,kind", [(1, 1, "tree"), (3, 5, "tree"), (2, 32, "tree"), (5, 33, "wild"), (2, 200, "tree"),
                                         (1, 1024, "tree"), (2, 1024, "chain"), (1, 700, "flat"), (70, 64, "wild")])
def test_tree(n, rows, kind):
    rng = random.Random(rows)
    lens = [rng.randint(0, 300) for _ in range(n)]
    kp = hold(new_pages(pages=20 * n, seqs=n + 1, blocks=19), lens)
    parent = [list(range(-1, rows - 1)) if kind == "chain" else [-1] * rows if kind == "flat" else
              random_tree(rng, rows, kind == "wild") for _ in range(n)]
    seqs = rng.sample(range(n), n)
    if n > 2:
        seqs[1], seqs[2] = n + 1, -1                                  # no sequences: as empty ones
    w = (rows + 31) // 32
    for counts in (None, [rng.randint(-1, rows + 1) for _ in range(n)]):
        mask, pos = torch.full((n, rows, w), 7, dtype=torch.int32, device=DEV), torch.full((n, rows), 7, dtype=torch.int32, device=DEV)
        P.kv_pages_tree(kp, ints(seqs), ints(parent), mask, pos, n_rows=None if counts is None else ints(counts))
        only = torch.zeros_like(mask)
        P.kv_pages_tree(kp, ints(seqs), ints(parent), only, n_rows=None if counts is None else ints(counts))
        for b, s in enumerate(seqs):
            c = rows if counts is None else min(max(counts[b], 0), rows)
            see = sees(parent[b][:c])
            held = lens[s] if 0 <= s < n else 0
            assert np.array_equal(mask[b, :c].cpu().numpy(), words(see, rows)) and torch.equal(only[b, :c], mask[b, :c])
            assert pos[b, :c].tolist() == [held - c + int(x) - 1 for x in see.sum(1)]
            assert bool((mask[b, c:] == 7).all()) and bool((pos[b, c:] == 7).all()) and not only[b, c:].any()


# ---------------------------------------------------------------- attention

def masks(rng, n, rows, kind):
    """Per entry [rows][rows] of what is seen: trees, or any pattern with rows that see nothing."""
    out = []
    for _ in range(n):
        if kind == "tree":
            out.append(sees(random_tree(rng, rows)))
        else:
            m = np.array([[rng.random() < 0.3 for _ in range(rows)] for _ in range(rows)], dtype=bool).reshape(rows, rows)
            m[rng.randrange(rows)] = False
            out.append(m)
    return out


def bits_of(see, rows):
    return torch.from_numpy(np.stack([words(m, rows) for m in see])).to(DEV)


def run_tree(kp, layer, seqs, q, counts, see, **kw):
    n, rows, heads, hd = q.shape
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=DEV)
    ws = torch.full((P.kv_pages_attention_workspace_bytes(kp, n, rows, heads),), 255, dtype=torch.uint8, device=DEV)
    P.kv_pages_attention_tree(kp, layer, ints(seqs), q, out, bits_of(see, rows), ws, n_rows=None if counts is None else ints(counts), **kw)
    return out


def near(a, b, v_max):
    """Of two ways to the same bf16 output: each is off by the rounding of its
    weights (2^-11) and sums (below 2^-10 here) of values up to v_max, and half
    a step of bf16 (2^-8)."""
    return np.abs(a - b) <= 2 * (v_max * (2.0 ** -11 + 2.0 ** -10) + np.abs(b) * 2.0 ** -8)


def check_tree(kp, layer, seqs, q, counts, see, scale=None, **kw):
    """Tolerances as in check_attention of the attention without trees."""
    n, rows, heads, hd = q.shape
    got = host(run_tree(kp, layer, seqs, q, counts, see, scale=scale, **kw))
    counts = [rows] * n if counts is None else [min(max(c, 0), rows) for c in counts]
    none = np.zeros((0, kp.n_kv_heads, hd))
    kv = [gather(kp, layer, s) if 0 <= s < kp.table.shape[0] else (none, none) for s in seqs]
    want, mass, size = attend_tree(host(q), [k for k, _ in kv], [v for _, v in kv], counts, see,
                                   hd ** -0.5 if scale is None else scale)
    longest = max(k.shape[0] for k, _ in kv)
    tol = mass * 2.0 ** -24 * (2 * (hd + 4) * size + longest + 64)
    if q.dtype == BF16:
        tol += mass * 2.0 ** -11 + np.abs(want) * 2.0 ** -8
    for b, c in enumerate(counts):
        assert np.all(got[b, c:] == 7.0)                              # rows past the count as they were
        diff, t = np.abs(got[b, :c] - want[b, :c]), tol[b, :c] + 1e-30
        assert np.all(diff <= t), (b, float(np.max(diff / t)))


@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("dtype,hd,page,heads,kv,rows,lens", [
    (BF16, 64, 16, 1, 1, 1, [1]),
    (BF16, 128, 64, 4, 4, 1, [1, 63, 64, 65, 200]),
    (BF16, 64, 16, 8, 2, 2, [0, 5, 300, 1000]),                       # an empty sequence
    (BF16, 128, 128, 8, 1, 3, [2, 400, 129]),                         # fewer positions than rows
    (BF16, 128, 32, 2, 2, 33, [33, 60, 500, 7]),
    (BF16, 64, 256, 2, 1, 65, [300, 1]),
    (BF16, 128, 16, 2, 2, 130, [130, 260, 97]),
    (BF16, 64, 32, 6, 2, 50, [700, 50, 51]),
    (BF16, 128, 16, 1, 1, 300, [1000, 310]),                          # trees of several words and tiles
    (F32, 64, 16, 2, 2, 1, [1, 40, 500]),
    (F32, 128, 32, 4, 2, 17, [17, 200, 9]),
    (F32, 64, 64, 3, 3, 70, [70, 333, 0]),
    (F32, 128, 256, 1, 1, 150, [400]),
])
def test_tree_attention(dtype, hd, page, heads, kv, rows, lens, kind):
    kp = hold(new_pages(pages=2 + sum(-(-m // page) for m in lens), heads=kv, page=page, hd=hd, seqs=len(lens),
                        blocks=max(1, -(-max(lens) // page)), dtype=dtype), lens)
    poison(kp)
    n = len(lens)
    seqs = list(range(n))[::-1]
    q, rng = queries(n, rows, heads, hd, dtype), random.Random(rows)
    check_tree(kp, 1, seqs, q, None, masks(rng, n, rows, kind), max_len=max(lens))
    check_tree(kp, 1, seqs, q, [max(0, rows - 2 * i) for i in range(n)], masks(rng, n, rows, kind), max_len=max(lens))


@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("case", [c for c in WAYS if c[6] > 1], ids=str)
def test_tree_attention_on_every_launch(case, kind):
    """Trees behind a prefix, one that reaches back into it and one of an empty sequence among them."""
    dtype, hd, page, heads, kv, n, rows, prefix, tail = case[:9]
    kp, seqs, lens = batch(case)
    poison(kp)
    assert division(P.kv_pages_attention_plan(kp, n, rows, heads, prefix, max(lens))) == case[9:]
    rng = random.Random(n)
    q = queries(n, rows, heads, hd, TYPES[dtype])
    counts = None if kind == "tree" else [max(0, rows - i % 4 * (rows // 3)) for i in range(n)]
    check_tree(kp, 1, seqs, q, counts, masks(rng, n, rows, kind), prefix_seq=0, shared_len=prefix, max_len=max(lens))


@pytest.mark.parametrize("dtype,hd,page,heads,kv,rows,prefix,lens", [
    (BF16, 64, 32, 2, 2, 7, 96, [100, 20, 0, 97]),                    # trees that begin inside the prefix
    (BF16, 128, 16, 4, 1, 40, 15, [60, 61]),                          # no whole page is shared
    (BF16, 64, 128, 2, 2, 3, 1024, [1027, 1024]),
    (BF16, 128, 64, 4, 4, 32, 512, [544] * 5),
    (F32, 64, 16, 2, 2, 19, 203, [222, 260, 333]),
])
def test_tree_attention_over_a_shared_prefix(dtype, hd, page, heads, kv, rows, prefix, lens):
    kp = shared_batch(dtype, hd, page, kv, prefix, lens)
    poison(kp)
    n, rng = len(lens), random.Random(1)
    seqs, q, see = list(range(1, n + 1)), queries(n, rows, heads, hd, dtype), masks(rng, len(lens), rows, "tree")
    for kw in (dict(shared_len=prefix, max_len=max(lens)), dict(shared_len=prefix + 1000, max_len=1),
               dict(shared_len=max(1, prefix // 2)), dict(shared_len=prefix, max_len=20000)):
        check_tree(kp, 0, seqs, q, None, see, prefix_seq=0, **kw)
    # entries that are no sequence, twice the same one, and the prefix itself
    some = [-1, 1, 1, 99, 0][:max(n, 2)]
    check_tree(kp, 0, some, queries(len(some), rows, heads, hd, dtype), None, masks(rng, len(some), rows, "any"), prefix_seq=0,
               shared_len=prefix, max_len=max(lens))


@pytest.mark.parametrize("what", ["inf", "nan", "lowest"])
@pytest.mark.parametrize("case", [c for c in WAYS if c[6] > 1] + [
    ("bf16", 64, 16, 2, 2, 2, 5, 0, 60, 0, 0, 16, False, False), ("bf16", 128, 16, 2, 2, 2, 20, 0, 60, 0, 0, 32, False, False),
    ("bf16", 128, 16, 2, 2, 2, 70, 0, 300, 0, 0, 128, False, False), ("f32", 128, 16, 2, 2, 2, 9, 0, 60, 0, 0, 16, False, False),
], ids=str)
def test_values_that_a_row_does_not_see(case, what):
    """Keys and values of one row of each tree made infinite, no number or the
    lowest of their type: rows that do not see it are as before (fp32: bit for
    bit; the exponent reference of bf16 rows is that of 32 together), outputs of
    the others are infinite or none as the sum is."""
    dtype, hd, page, heads, kv, n, rows, prefix, tail = case[:9]
    lens = [prefix + rows + tail + 3 * b for b in range(n)]
    kp = shared_batch(TYPES[dtype], hd, page, kv, prefix, lens)
    poison(kp)
    seqs, rng = list(range(1, n + 1)), random.Random(rows)
    q, see = queries(n, rows, heads, hd, TYPES[dtype]), masks(rng, n, rows, "tree")
    for m in see:
        m[rows - 1, 0] = False                                        # a row that does not see the first
    kw = dict(prefix_seq=0, shared_len=prefix, max_len=max(lens))
    clean = host(run_tree(kp, 1, seqs, q, None, see, **kw))
    assert np.isfinite(clean).all()
    v_max = float(kp.vt[1].nan_to_num(nan=0.0).abs().max())
    table = kp.table.tolist()
    for b, m in enumerate(lens):
        at, slot = table[b + 1][(m - rows) // page], (m - rows) % page
        if what == "lowest":
            kp.vt[1, at, :, :, slot] = torch.finfo(kp.vt.dtype).min
        else:
            kp.vt[1, at, :, :, slot] = float(what)
            kp.vt[1, at, :, 1::2, slot] = -float(what)
            if what == "inf" and rows > 2:                            # the other sign in the next row: they meet in a NaN
                kp.vt[1, table[b + 1][(m - rows + 1) // page], :, 4, (m - rows + 1) % page] = float("-inf")
        if what == "nan":
            kp.k[1, at, :, slot] = float("nan")
    got = host(run_tree(kp, 1, seqs, q, None, see, **kw))
    first = np.stack([m[:, 0] for m in see])[:, :, None, None]
    second = np.stack([m[:, min(1, rows - 1)] for m in see])[:, :, None, None] & (what == "inf" and rows > 2)
    with np.errstate(invalid="ignore"):
        add = np.zeros_like(clean)
        if what == "nan":
            add += np.where(first, np.nan, 0)
        elif what == "inf":
            add[..., 0::2] += np.where(first, np.inf, 0)
            add[..., 1::2] -= np.where(first, np.inf, 0)
            add[..., 4:5] -= np.where(second, np.inf, 0)
        want = clean + add
        # rows that see the lowest value: finite in bf16, past fp32 before the
        # division (weights of up to 2^15 times 2^128)
        low = np.broadcast_to(first & (what == "lowest"), got.shape)
        assert dtype == "f32" or np.isfinite(got[low]).all()
        kinds = lambda x: np.select([np.isnan(x), np.isposinf(x), np.isneginf(x)], [1, 2, 3], 0)
        wrong = int((kinds(got) != kinds(want))[~low].sum())
        assert wrong == 0
        far = int(((got != clean) & ~(near(got, clean, v_max) & (dtype == "bf16")) & np.isfinite(add) & ~low).sum())
        assert far == 0


@pytest.mark.parametrize("dtype,rows,lens", [(BF16, 5, [40, 70]), (BF16, 20, [300, 33]), (BF16, 140, [500, 200]), (F32, 7, [90, 17])])
def test_a_chain_is_causal(dtype, rows, lens):
    """A tree without branches sees what causal rows see."""
    kp = hold(new_pages(pages=90, seqs=2, blocks=32, dtype=dtype), lens)
    q = queries(2, rows, 2, 64, dtype)
    see = [sees(list(range(-1, rows - 1)))] * 2
    got = run_tree(kp, 0, [0, 1], q, None, see)
    out = torch.zeros_like(q)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, 2, rows, 2), dtype=torch.uint8, device=DEV)
    P.kv_pages_attention(kp, 0, ints([0, 1]), q, out, ws, causal=True)
    if dtype == BF16:
        assert near(host(got), host(out), float(kp.vt.abs().max())).all()
    else:
        # sums of up to 500 keys and scores of up to 40, as in check_attention
        assert bool(((got - out).abs() <= 2 * kp.vt.abs().max() * 2.0 ** -24 * (2 * 68 * 40 + 564)).all())


def test_tree_attention_strides():
    kp = hold(new_pages(seqs=3, pages=60, blocks=20, heads=4), [300, 64, 290])
    q = normal(3, 8, 11, 64, seed=3).permute(0, 2, 1, 3)
    see = masks(random.Random(2), 3, 11, "tree")
    want = run_tree(kp, 1, [0, 1, 2], q, None, see)
    buf = torch.zeros(3, 8, 15, 80, dtype=BF16, device=DEV)
    out = buf[:, :, 2:13, 8:72].permute(0, 2, 1, 3)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, 3, 11, 8), dtype=torch.uint8, device=DEV)
    P.kv_pages_attention_tree(kp, 1, ints([0, 1, 2]), q, out, bits_of(see, 11), ws)
    assert torch.equal(out, want)
    buf[:, :, 2:13, 8:72] = 0
    assert not buf.any()


# ---------------------------------------------------------------- acceptance

class Drafts(Both):
    """The library's cache and the host model with acceptance, held against one another after every call."""

    def __init__(self, **kw):
        super().__init__(**kw)
        h, self.h = self.h, HostDrafts(self.d.k.shape[1], self.d.page_len, *self.d.table.shape)
        self.h.refs, self.h.table, self.h.len = h.refs, h.table, h.len

    def accept(self, seqs, counts, max_rows, paths, max_path, junk=-9):
        want = self.h.accept(seqs, counts, max_rows, paths, max_path)
        if want == OK:
            for (a, x), (b, y) in self.h.rows_moved:                  # in order: no place is read after it is filled
                self.k[:, b, :, y], self.vt[:, b, :, :, y] = self.k[:, a, :, x], self.vt[:, a, :, :, x]
        n = len(seqs)
        ws = torch.full((P.kv_pages_accept_workspace_bytes(self.d, n, max_path),), 255, dtype=torch.uint8, device=DEV)
        rows = [p[:max_path] + [junk] * (max_path - len(p)) for p in paths]
        P.kv_pages_accept(self.d, ints(seqs), ints(rows), ints([len(p) for p in paths]), self.status, ws, rows=max_rows,
                          n_rows=None if counts == [max_rows] * n else ints(counts))
        assert self.status.item() == want, (seqs, counts, paths)
        self.check()
        return want


@pytest.mark.parametrize("seed,kw", [
    (0, {}),
    (1, dict(page=32, hd=128, dtype=torch.float32, pages=23)),
    (2, dict(layers=1, heads=1, pages=1100, seqs=40, blocks=70)),
    (3, dict(page=256, heads=3, pages=9, blocks=3, hd=128)),
    (4, dict(pages=2500, seqs=600, blocks=60, heads=1, layers=1)),    # tables past what one workgroup clears
    (5, dict(layers=3, heads=8, hd=128)),                             # rows past what one workgroup moves
    (6, dict(layers=4, heads=9, hd=128, dtype=torch.float32)),
    (7, dict(layers=4, heads=7, dtype=torch.float32)),
])
def test_random_acceptances(seed, kw):
    rng = random.Random(seed)
    both = Drafts(seed=seed, **kw)
    n_seqs, page = both.d.table.shape[0], both.d.page_len
    seen = set()
    for _ in range(40):
        held = [s for s in range(n_seqs) if both.h.len[s]]
        empty = [s for s in range(n_seqs) if not both.h.len[s]]
        what = rng.choice(["grow", "fork", "accept", "accept"])
        if what == "grow":
            seqs = rng.sample(range(n_seqs), rng.randint(1, n_seqs))
            both.call("grow", seqs, [rng.choice([1, 5, page, 2 * page + 3]) for _ in seqs])
        elif what == "fork" and held and empty:
            dst = rng.sample(empty, rng.randint(1, min(3, len(empty))))
            both.call("fork", [rng.choice(held) for _ in dst], dst)
        elif what == "accept" and held:
            seqs = rng.sample(held, rng.randint(1, len(held)))
            counts = [rng.randint(0, min(both.h.len[s], 40)) for s in seqs]
            paths = [sorted(rng.sample(range(c), min(c, rng.randint(0, 12)))) for c in counts]
            seen.add(both.accept(seqs, counts, 40, paths, 12))
    assert OK in seen


def test_acceptance_errors_change_nothing():
    both = Drafts(pages=12, page=16, seqs=6, blocks=5)
    assert both.call("grow", [0, 1], [40, 32]) == OK
    assert both.accept([0, 0], [5, 5], 5, [[1], [1]], 2) == ESEQ
    assert both.accept([0, 6], [5, 5], 5, [[1], [1]], 2) == ESEQ
    assert both.accept([-1], [5], 5, [[1]], 2) == ESEQ
    assert both.accept([0], [6], 5, [[1]], 2) == ELEN                 # more rows than there may be
    assert both.accept([0], [-1], 5, [[]], 2) == ELEN
    assert both.accept([0], [41], 60, [[1]], 2) == ELEN               # more than it holds
    assert both.accept([2], [1], 5, [[]], 2) == ELEN
    assert both.accept([0], [3], 5, [[0, 1, 2, 2]], 4) == ELEN        # a path longer than its rows
    assert both.accept([0, 1], [9, 9], 9, [[1, 4], [3, 9]], 3) == EPATH
    assert both.accept([0], [9], 9, [[4, 4]], 3) == EPATH
    assert both.accept([0], [9], 9, [[5, 4]], 3) == EPATH
    assert both.accept([0], [9], 9, [[-1, 4]], 3) == EPATH
    assert both.accept([1, 0, 0], [9, 9, 9], 9, [[4, 4], [1], [1]], 3) == ESEQ      # the lowest code
    assert both.call("fork", [1, 1], [2, 3]) == OK                    # whole pages, held three times
    assert both.accept([1], [10], 10, [[4]], 3) == ESHARED            # into a shared page
    assert both.accept([1], [10], 10, [[0, 1]], 3) == ESHARED         # cut inside one
    assert both.accept([1], [10], 10, [[4, 4]], 3) == ESHARED         # lower than the path's
    assert both.accept([2], [16], 16, [[]], 3) == OK                  # cut between pages
    assert both.accept([1], [10], 10, [list(range(10))], 10) == OK    # nothing moves, nothing is cut
    assert both.accept([0, 3], [30, 0], 30, [[0, 7, 8, 20, 29], []], 7) == OK
    assert both.accept([0], [15], 15, [[]], 1) == OK                  # nothing is left


def test_long_paths():
    """Paths of many batches of rows, over pages and back by one."""
    for dtype, hd, heads in ((BF16, 128, 2), (F32, 64, 2), (BF16, 64, 11), (F32, 128, 11)):
        both = Drafts(pages=160, page=16, seqs=3, blocks=70, dtype=dtype, hd=hd, heads=heads)
        assert both.call("grow", [0, 1, 2], [1040, 1030, 17]) == OK
        rng = random.Random(2)
        paths = [list(range(1, 1024)), sorted(rng.sample(range(1024), 500)), [16]]
        assert both.accept([0, 1, 2], [1024, 1024, 17], 1024, paths, 1023) == OK


# ---------------------------------------------------------------- together

def round_of(kp, st, seqs, add, parent, mask, pos, qkv, rot, q, out, ws, path, n_path, ws2):
    rows, kv = parent.shape[1], kp.n_kv_heads
    P.kv_pages_grow(kp, seqs, add, st[0:1])
    P.kv_pages_tree(kp, seqs, parent, mask, pos)
    heads = q.shape[2]
    for layer in range(kp.k.shape[0]):
        x = qkv[layer]
        P.kv_pages_append(kp, layer, seqs, x[:, :, heads:heads + kv], x[:, :, heads + kv:], rot, q=x[:, :, :heads], q_out=q, pos=pos)
        P.kv_pages_attention_tree(kp, layer, seqs, q, out[layer], mask, ws)
    P.kv_pages_accept(kp, seqs, path, n_path, st[1:2], ws2, rows=rows)


def test_drafts_verified_as_tokens_one_after_another():
    """Every path of a tree attends as its tokens do, appended in turn; what is
    accepted leaves the cache as if those tokens alone had been appended."""
    kp = hold(new_pages(pages=40, seqs=3, blocks=10, heads=2), [37])
    rows, heads, rot = 9, 4, new_rotary(64, 32, "pairs", True)
    parent = [-1, 0, 0, 1, 2, 2, 4, 3, 5]
    st = ints([9, 9])
    qkv = normal(2, 1, rows, heads + 4, 64, seed=12)
    seq = ints([0])
    mask, pos = torch.zeros(1, rows, 1, dtype=torch.int32, device=DEV), torch.zeros(1, rows, dtype=torch.int32, device=DEV)
    q, out = torch.zeros(1, rows, heads, 64, dtype=BF16, device=DEV), torch.zeros(2, 1, rows, heads, 64, dtype=BF16, device=DEV)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, 1, rows, heads), dtype=torch.uint8, device=DEV)
    path = [0, 2, 4, 6]
    ws2 = torch.empty(P.kv_pages_accept_workspace_bytes(kp, 1, 4), dtype=torch.uint8, device=DEV)
    k0, vt0 = kp.k.clone(), kp.vt.clone()
    round_of(kp, st, seq, ints([rows]), ints([parent]), mask, pos, qkv, rot, q, out, ws, ints([path]), ints([4]), ws2)
    assert st.tolist() == [0, 0] and kp.len[0].item() == 41
    one = hold(new_pages(pages=40, seqs=3, blocks=10, heads=2), [37])
    one.k.copy_(k0)
    one.vt.copy_(vt0)
    for j, r in enumerate(path):
        P.kv_pages_grow(one, seq, ints([1]), st[0:1])
        for layer in range(2):
            x = qkv[layer][:, r:r + 1]
            q1, o1 = torch.zeros(1, 1, heads, 64, dtype=BF16, device=DEV), torch.zeros(1, 1, heads, 64, dtype=BF16, device=DEV)
            P.kv_pages_append(one, layer, seq, x[:, :, heads:heads + 2], x[:, :, heads + 2:], rot, q=x[:, :, :heads], q_out=q1)
            P.kv_pages_attention(one, layer, seq, q1, o1, ws)
            assert near(host(out[layer][:, r:r + 1]), host(o1), float(kp.vt.abs().max())).all()
    for layer in range(2):
        for a, b in zip(gather(kp, layer, 0), gather(one, layer, 0)):
            assert np.array_equal(a, b)


def test_rounds_captured_and_replayed():
    """Grow, tree, append, attend and accept in one graph, replayed between the
    same calls made eagerly on another stream: all of them give the same."""
    n, rows, heads = 5, 21, 4
    kp = hold(new_pages(pages=80, seqs=n, blocks=12, heads=2), [37, 16, 0, 90, 5])
    rot, rng = new_rotary(64, norm=True), random.Random(7)
    st, seqs, add = ints([9, 9]), ints([3, 0, 4, 1, 2]), ints([rows] * n)
    parent = ints([random_tree(rng, rows) for _ in range(n)])
    path, n_path = ints([[0, 1, 7, 11]] * n), ints([4, 2, 0, 3, 1])
    mask, pos = torch.zeros(n, rows, 1, dtype=torch.int32, device=DEV), torch.zeros(n, rows, dtype=torch.int32, device=DEV)
    qkv = normal(2, n, rows, heads + 4, 64, seed=12)
    q, out = torch.zeros(n, rows, heads, 64, dtype=BF16, device=DEV), torch.zeros(2, n, rows, heads, 64, dtype=BF16, device=DEV)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, n, rows, heads), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty(P.kv_pages_accept_workspace_bytes(kp, n, 4), dtype=torch.uint8, device=DEV)
    args = (kp, st, seqs, add, parent, mask, pos, qkv, rot, q, out, ws, path, n_path, ws2)
    arrays = (kp.k, kp.vt, kp.refs, kp.table, kp.len)
    start = [t.clone() for t in arrays]

    def reset():
        for t, x in zip(arrays, start):
            t.copy_(x)
        for t in (mask, pos, q, out):
            t.zero_()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        round_of(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        round_of(*args)
    for replay in range(3):
        qkv.normal_()
        parent.copy_(ints([random_tree(rng, rows) for _ in range(n)]))
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert st.tolist() == [0, 0] and kp.len.tolist() == [37 + 2, 16 + 3, 0 + 1, 90 + 4, 5 + 0]
        got = [t.clone() for t in arrays + (mask, pos, out)]
        reset()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            round_of(*args)
        torch.cuda.synchronize()
        for a, b in zip(got, arrays + (mask, pos, out)):
            assert torch.equal(a, b)
        for b, p in enumerate(parent.tolist()):
            assert np.array_equal(mask[b].cpu().numpy(), words(sees(p), rows))


def test_refusals():
    kp = hold(new_pages(seqs=3), [40, 20, 0])
    rot = new_rotary(64)
    q = normal(2, 3, 2, 64)
    out, ws = torch.empty_like(q), torch.empty(P.kv_pages_attention_workspace_bytes(kp, 2, 3, 2), dtype=torch.uint8, device=DEV)
    two, st, mask = ints([0, 1]), ints([0]), torch.zeros(2, 3, 1, dtype=torch.int32, device=DEV)
    parent, path = ints([[-1, 0, 1]] * 2), ints([[0, 1]] * 2)
    ws2 = torch.empty(P.kv_pages_accept_workspace_bytes(kp, 2, 2), dtype=torch.uint8, device=DEV)
    bad = [
        lambda: P.Rotary(96, device=DEV),
        lambda: P.Rotary(64, dim=24, device=DEV),
        lambda: P.Rotary(64, layout="quarters", device=DEV),
        lambda: P.Rotary(64, scaling="log", device=DEV),
        lambda: P.Rotary(64, freq=[1.0, 2.0], device=DEV),
        lambda: P.Rotary(64, q_gain=torch.ones(64, device=DEV), device=DEV),
        lambda: P.Rotary(64, norm=True, q_gain=torch.ones(64, dtype=BF16, device=DEV), device=DEV),
        lambda: P.Rotary(64, norm=True, k_gain=torch.ones(64), device=DEV),
        lambda: P.Rotary(64, norm=True, k_gain=torch.ones(32, device=DEV), device=DEV),
        lambda: P.rotary_rows(rot, q.half(), out),
        lambda: P.rotary_rows(rot, q, out.float()),
        lambda: P.rotary_rows(rot, q, out[:, :2]),
        lambda: P.rotary_rows(rot, q, None),
        lambda: P.rotary_rows(rot, q[..., :32], out[..., :32]),
        lambda: P.rotary_rows(rot, q, out, q[:, :2], out[:, :2]),
        lambda: P.rotary_rows(rot, q, out, pos=ints([[1, 2]] * 2)),
        lambda: P.rotary_rows(rot, q, out, pos=ints([[1, 2, 3]] * 2).long()),
        lambda: P.rotary_rows(rot, q, out, pos=ints([[1, 2, 3]] * 2).cpu()),
        lambda: P.rotary_rows(rot, q, out, n_rows=ints([1])),
        lambda: P.rotary_rows(rot, q.transpose(2, 3).contiguous().transpose(2, 3), out),
        lambda: P.rotary_rows(rot, q.cpu(), out.cpu()),
        lambda: P.kv_pages_append(kp, 0, two, q, q[:, :2], rot),
        lambda: P.kv_pages_append(kp, 0, two, q[:, :, :1], q[:, :, :1], rot),
        lambda: P.kv_pages_append(kp, 0, two, q, q, rot, q=q[:, :2], q_out=out[:, :2]),
        lambda: P.kv_pages_append(kp, 0, two, q, q, rot, q=q),
        lambda: P.kv_pages_append(kp, 0, two, q.float(), q.float(), rot),
        lambda: P.kv_pages_append(kp, 0, two, q, q, rot, pos=ints([[1, 2]] * 2)),
        lambda: P.kv_pages_tree(kp, two, parent, mask[:, :2]),
        lambda: P.kv_pages_tree(kp, two, parent.long(), mask),
        lambda: P.kv_pages_tree(kp, two, parent, mask, pos=ints([1, 2])),
        lambda: P.kv_pages_tree(kp, ints([0]), parent, mask),
        lambda: P.kv_pages_attention_tree(kp, 0, two, q, out, mask[:1], ws),
        lambda: P.kv_pages_attention_tree(kp, 0, two, q, out, mask.long(), ws),
        lambda: P.kv_pages_attention_tree(kp, 0, two, q, out[:, :2], mask, ws),
        lambda: P.kv_pages_attention_tree(kp, 0, two, q, out, mask.cpu(), ws),
        lambda: P.kv_pages_accept(kp, two, path, ints([1]), st, ws2, rows=3),
        lambda: P.kv_pages_accept(kp, ints([0]), path, two, st, ws2, rows=3),
        lambda: P.kv_pages_accept(kp, two, path.long(), two, st, ws2, rows=3),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    refused = [
        lambda: P.rotary_rows(rot, q, out[:, :1].expand(2, 3, 2, 64)),
        lambda: P.rotary_rows(rot, q, q.as_strided(q.shape, (384, 64, 192, 1))),
        lambda: P.kv_pages_append(kp, 2, two, q, q, rot),
        lambda: P.kv_pages_append(kp, 0, two, normal(2, 3, 2, 64), q, P.Rotary(128, device=DEV)),
        lambda: P.kv_pages_attention_tree(kp, 2, two, q, out, mask, ws),
        lambda: P.kv_pages_attention_tree(kp, 0, two, q, out, mask, ws, shared_len=-1),
        lambda: P.kv_pages_attention_tree(kp, 0, two, q, out, mask, ws, scale=0.0),
        lambda: P.kv_pages_attention_tree(kp, 0, two, q, out, mask, ws[1:]),
        lambda: P.kv_pages_accept(kp, two, path, two, st, ws2[:8], rows=3),
        lambda: P.kv_pages_accept(kp, two, path, two, st, ws2, rows=0),
    ]
    before = [t.clone() for t in (kp.k, kp.vt, kp.refs, kp.table, kp.len, q)]
    for call in refused:
        with pytest.raises(P.binding.DllmError):
            call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, (kp.k, kp.vt, kp.refs, kp.table, kp.len, q)))
