"""Rotations and drafted trees: refusals on the host before any device call, the
frequencies, and the host model that the GPU tests compare with (no GPU)."""
import ctypes as C
import os
import random

import numpy as np
import pytest

from tests.drafts_model import EPATH, HostDrafts, attend_tree, frequencies, rotate, sees, words
from tests.pages_model import OK, ESEQ, ELEN, ESHARED, attend
from tests.test_pages_cpu import BAD_PAGES, FAKE, pages

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_11742_amd", "libdllm_rps.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libdllm_rps.so not built")


@pytest.fixture(scope="module")
def abi():
    from paper_2608_11742_amd import _abi
    return _abi, _abi.load()


def rotary(_abi, **kw):
    d = dict(freq=FAKE, q_gain=None, k_gain=None, head_dim=64, dim=64, layout=0, norm=0, amplitude=1.0, eps=1e-5)
    d.update(kw)
    return _abi.RotaryC(*[d[f] for f, _ in _abi.RotaryC._fields_])


BAD_ROTARY = [(dict(head_dim=96, dim=32), 2), (dict(dim=-16), 2), (dict(dim=80), 2), (dict(dim=24), 2), (dict(layout=2), 1),
              (dict(layout=-1), 1), (dict(freq=None), 1), (dict(freq=FAKE + 4), 1), (dict(amplitude=float("nan")), 1),
              (dict(amplitude=float("inf")), 1), (dict(norm=1, eps=0.0), 1), (dict(norm=1, eps=float("inf")), 1),
              (dict(norm=1, eps=float("nan")), 1), (dict(norm=1, q_gain=FAKE + 4), 1), (dict(norm=1, k_gain=FAKE + 8), 1)]


@needs_lib
@pytest.mark.parametrize("field,value,status", BAD_PAGES)
def test_pages_are_checked(abi, field, value, status):
    _abi, lib = abi
    p = C.byref(pages(_abi, **{field: value}))
    r, rot = C.byref(_abi.Rows(FAKE, 64, 64, 64)), C.byref(rotary(_abi))
    assert lib.kv_pages_append(p, 0, FAKE, 1, 1, None, rot, None, 0, None, None, r, r, None) == status
    assert lib.kv_pages_tree(p, FAKE, 1, 1, None, FAKE, FAKE, None, None) == status
    assert lib.kv_pages_attention_tree(p, 0, FAKE, 1, 1, None, 2, r, r, FAKE, 0, 0, 1, 1.0, FAKE, 1 << 40, None) == status
    assert lib.kv_pages_accept(p, FAKE, 1, 1, None, FAKE, 1, FAKE, FAKE, FAKE, 1 << 30, None) == status
    assert lib.kv_pages_accept_workspace_bytes(p, 1, 1) == 0


@needs_lib
@pytest.mark.parametrize("kw,status", BAD_ROTARY)
def test_rotations_are_checked(abi, kw, status):
    _abi, lib = abi
    rot, r = C.byref(rotary(_abi, **kw)), C.byref(_abi.Rows(FAKE, 64, 64, 64))
    assert lib.rotary_rows(rot, 1, None, 0, 1, 1, None, 1, r, r, 0, None, None, None) == status
    p = C.byref(pages(_abi))
    assert lib.kv_pages_append(p, 0, FAKE, 1, 1, None, rot, None, 0, None, None, r, r, None) == status
    assert lib.dllm_last_error()


@needs_lib
def test_rows_are_checked(abi):
    _abi, lib = abi
    R = _abi.Rows
    good = R(FAKE, 1024, 256, 64)

    def turn(rot=rotary(_abi), dtype=1, n=2, rows=4, hq=4, q=good, qo=R(1 << 20, 1024, 256, 64), hk=0, k=None, ko=None, n_rows=None):
        ref = lambda x: None if x is None else C.byref(x)
        return lib.rotary_rows(ref(rot), dtype, None, 0, n, rows, n_rows, hq, ref(q), ref(qo), hk, ref(k), ref(ko), None)

    assert turn(rot=None) == 1 and turn(dtype=2) == 3 and turn(dtype=-1) == 3
    assert turn(n=0) == 2 and turn(n=1025) == 2 and turn(rows=0) == 2 and turn(rows=(1 << 20) + 1) == 2
    assert turn(hq=0) == 2 and turn(hq=-1) == 2 and turn(hq=1025) == 2 and turn(hk=-1) == 2 and turn(hk=1025) == 2
    assert turn(n=1024, rows=1 << 10, hq=65) == 2                      # past KV_MAX_HEAD_ROWS
    assert turn(q=None) == 1 and turn(qo=None) == 1 and turn(hk=1) == 1
    for bad, status in [(R(None, 64, 64, 64), 1), (R(FAKE + 2, 64, 64, 64), 1), (R(FAKE, 64, 60, 64), 1),
                        (R(FAKE, -64, 64, 64), 2), (R(FAKE, 64, 64, (1 << 40) + 8), 2)]:
        assert turn(q=bad) == status and turn(qo=bad) == status
        assert turn(hk=2, k=bad, ko=good) == status and turn(hk=2, k=good, ko=bad) == status
    # rows of the output on one another, and in place at other strides
    for out in (R(1 << 20, 0, 256, 64), R(1 << 20, 1024, 0, 64), R(1 << 20, 1024, 256, 56), R(1 << 20, 512, 256, 64)):
        assert turn(qo=out) == 2
    assert turn(qo=R(1 << 20, 1024, 256, 56), n_rows=FAKE) == 2
    assert turn(qo=R(FAKE, 1024, 512, 64)) == 1 and turn(qo=R(FAKE, 2048, 256, 64)) == 1

    p = C.byref(pages(_abi))

    def append(pg=p, layer=0, seqs=FAKE, n=2, rows=4, rot=rotary(_abi), heads=0, q=None, qo=None, k=good, v=good):
        ref = lambda x: None if x is None else C.byref(x)
        return lib.kv_pages_append(pg, layer, seqs, n, rows, None, ref(rot), None, heads, ref(q), ref(qo), ref(k), ref(v),
                                   None)

    assert append(rot=None) == 1 and append(rot=rotary(_abi, head_dim=128)) == 2
    assert append(seqs=None) == 1 and append(n=0) == 2 and append(n=1025) == 2 and append(rows=0) == 2
    assert append(rows=(1 << 20) + 1) == 2 and append(layer=2) == 2 and append(layer=-1) == 2
    assert append(heads=-1) == 2 and append(heads=1025) == 2 and append(heads=2) == 1 and append(heads=2, q=good) == 1
    assert append(heads=4, q=good, qo=R(1 << 20, 1024, 128, 64)) == 2
    assert append(k=None) == 1 and append(v=None) == 1 and append(k=R(FAKE, 64, 60, 64)) == 1 and append(v=R(FAKE + 8, 64, 64, 64)) == 1


@needs_lib
def test_tree_arguments(abi):
    _abi, lib = abi
    p = C.byref(pages(_abi))
    top = _abi.KV_TREE_MAX_ROWS
    assert top == 1024

    def tree(seqs=FAKE, n=1, rows=4, parent=FAKE, mask=FAKE):
        return lib.kv_pages_tree(p, seqs, n, rows, None, parent, mask, None, None)

    assert tree(seqs=None) == 1 and tree(n=0) == 2 and tree(n=1025) == 2 and tree(parent=None) == 1 and tree(mask=None) == 1
    assert tree(rows=0) == 2 and tree(rows=top + 1) == 2
    good = _abi.Rows(FAKE, 1024, 128, 64)
    need = lib.kv_pages_attention_workspace_bytes(p, 2, 4, 4)

    def attend_(q=good, o=good, layer=0, n=2, rows=4, heads=4, mask=FAKE, prefix=0, shared=0, most=64, scale=1.0, ws=FAKE,
                size=need):
        return lib.kv_pages_attention_tree(p, layer, FAKE, n, rows, None, heads, C.byref(q), C.byref(o), mask, prefix,
                                           shared, most, scale, ws, size, None)

    assert attend_(mask=None) == 1 and attend_(rows=top + 1, size=1 << 40) == 2
    assert attend_(layer=2) == 2 and attend_(layer=-1) == 2 and attend_(rows=0) == 2 and attend_(n=0) == 2
    assert attend_(heads=3) == 2 and attend_(heads=0) == 2 and attend_(shared=-1) == 2 and attend_(most=-1) == 2
    assert attend_(prefix=4, shared=1) == 1 and attend_(prefix=-1, shared=1) == 1
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert attend_(scale=scale) == 1
    assert attend_(ws=None) == 1 and attend_(ws=FAKE + 4) == 1 and attend_(size=need - 1) == 4
    assert attend_(o=_abi.Rows(FAKE, 1024, 0, 64)) == 2 and b"kv_pages_attention_tree" in lib.dllm_last_error()
    assert attend_(q=_abi.Rows(FAKE + 2, 64, 64, 64)) == 1

    def accept(seqs=FAKE, n=2, rows=8, path=FAKE, max_path=4, n_path=FAKE, status=FAKE, ws=FAKE, size=2 * 4 * 4):
        return lib.kv_pages_accept(p, seqs, n, rows, None, path, max_path, n_path, status, ws, size, None)

    assert lib.kv_pages_accept_workspace_bytes(p, 2, 4) == 32
    for n, m in ((0, 1), (1025, 1), (1, 0), (1, top + 1)):
        assert lib.kv_pages_accept_workspace_bytes(p, n, m) == 0
    assert accept(seqs=None) == 1 and accept(n=0) == 2 and accept(n=1025) == 2 and accept(rows=0) == 2
    assert accept(rows=(1 << 20) + 1) == 2 and accept(path=None) == 1 and accept(n_path=None) == 1 and accept(status=None) == 1
    assert accept(max_path=0) == 2 and accept(max_path=top + 1) == 2
    assert accept(ws=None) == 1 and accept(ws=FAKE + 8) == 1 and accept(size=31) == 4


@needs_lib
@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling="linear", factor=8.0), dict(scaling="base", factor=4.0),
                                dict(scaling="ramp", factor=16.0, original_len=8192.0),
                                dict(scaling="ramp", factor=8.0, slow=0.0, fast=4.0), dict(scaling="ramp", factor=1.0)])
@pytest.mark.parametrize("dim", [2, 16, 48, 64, 128])
def test_frequencies(dim, kw):
    import paper_2608_11742_amd as P
    got, amplitude = P.dllm_rotary_frequencies(dim, **kw)
    want, w_amp = frequencies(dim, **kw)
    # a power and a few products of doubles on both sides
    assert np.allclose(got, want, rtol=64 * 2.0 ** -53, atol=0) and abs(amplitude - w_amp) <= w_amp * 2.0 ** -24
    plain = frequencies(dim, kw.get("base", 10000.0))[0]
    factor = kw.get("factor", 1.0)
    if kw.get("scaling") == "linear":
        assert np.allclose(got, plain / factor)
    elif kw.get("scaling") == "base" and dim > 2:
        assert got[0] == 1.0 and np.isclose(got[-1], plain[-1] / factor)
    elif kw.get("scaling") == "ramp":
        assert np.all(np.array(got) <= plain * (1 + 1e-12)) and np.all(np.array(got) >= plain / factor * (1 - 1e-12))
    else:
        assert np.allclose(got, plain)


@needs_lib
def test_frequencies_are_checked(abi):
    _abi, lib = abi
    freq, amp = (C.c_double * 64)(), C.c_float()

    def ask(dim=64, base=1e4, scaling=0, factor=2.0, length=4096.0, slow=1.0, fast=32.0, f=freq, a=C.byref(amp)):
        return lib.dllm_rotary_frequencies(dim, base, scaling, factor, length, slow, fast, f, a)

    nan, inf = float("nan"), float("inf")
    assert ask() == 0 and ask(factor=nan) == 0                         # plain: no factor
    assert ask(f=None) == 1 and ask(a=None) == 1 and ask(dim=0) == 2 and ask(dim=7) == 2 and ask(dim=-2) == 2
    for base in (0.0, -1.0, nan, inf):
        assert ask(base=base) == 1
    assert ask(scaling=4) == 1 and ask(scaling=-1) == 1
    for s in (1, 2, 3):
        for factor in (0.5, nan, inf, -2.0):
            assert ask(scaling=s, factor=factor) == 1
    for kw in (dict(length=0.0), dict(length=nan), dict(slow=-1.0), dict(slow=32.0), dict(fast=inf), dict(fast=nan)):
        assert ask(scaling=3, **kw) == 1


def test_host_rotation():
    """Both layouts turn pairs by the angle: lengths stay, differences of positions are all that products see."""
    rng = np.random.default_rng(0)
    x, y = rng.normal(size=(2, 1, 64))
    f, _ = frequencies(48)
    for pairs in (False, True):
        turn = lambda v, p: rotate(v[None], np.array([p]), f, 48, pairs)[0][0]
        assert np.allclose(np.linalg.norm(turn(x, 77)), np.linalg.norm(x))
        assert np.allclose((turn(x, 1000) * turn(y, 990)).sum(), (turn(x, 10) * turn(y, 0)).sum())
        assert np.array_equal(turn(x, 5)[:, 48:], x[:, 48:]) and np.allclose(turn(x, 0), x)
    a, _ = rotate(x[None], np.array([3]), f, 48, True)
    order = np.concatenate([np.arange(0, 48, 2), np.arange(1, 48, 2), np.arange(48, 64)])
    b, _ = rotate(x[None][..., order], np.array([3]), f, 48, False)
    assert np.allclose(a[..., order], b)
    n, _ = rotate(x[None], np.array([0]), f, 48, False, norm=True, gain=np.full(64, 2.0))
    assert np.isclose((n * n).mean(), 4.0, rtol=1e-4)


def test_host_trees():
    see = sees([-1, 0, 0, 1, 7, 3, -5, 6])                             # rows 4 and 6 name no earlier row: roots
    want = [{0}, {0, 1}, {0, 2}, {0, 1, 3}, {4}, {0, 1, 3, 5}, {6}, {6, 7}]
    assert [set(np.flatnonzero(r)) for r in see] == want
    w = words(sees([-1] + list(range(39))), 40)
    assert w.shape == (40, 2) and w[31, 0] == -1 and w[39, 1] == 255 and w[0].tolist() == [1, 0]
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(1, 4, 2, 8)), rng.normal(size=(7, 1, 8)), rng.normal(size=(7, 1, 8))
    chain = sees([-1, 0, 1, 2])
    for a, b in zip(attend_tree(q, [k], [v], [4], [chain], 0.3), attend(q, [k], [v], [4], True, 0.3)):
        assert np.allclose(a, b)
    out, _, _ = attend_tree(q, [k[:3]], [v[:3]], [4], [np.eye(4, dtype=bool)], 0.3)   # row 0 has no position
    assert not out[0, 0].any() and np.allclose(out[0, 3], v[2, 0])


def test_host_acceptance_keeps_the_tables_sound():
    import copy
    rng = random.Random(5)
    h = HostDrafts(16, 16, 6, 6)
    assert h.grow([0], [32]) == OK and h.fork([0], [1]) == OK
    codes = {h.accept([0], [20], 28, [[3]], 4), h.accept([0], [20], 28, [[0, 1]], 4)}
    assert codes == {ESHARED} and h.accept([0], [20], 28, [[0, 1, 2, 3]], 4) == OK      # up to the page's end: nothing moves or is cut
    for _ in range(600):
        was = copy.deepcopy((h.refs, h.table, h.len))
        seqs = [rng.randrange(7) for _ in range(rng.randint(1, 3))]
        what = rng.choice(["grow", "fork", "free", "accept", "accept"])
        if what == "grow":
            code = h.grow(seqs, [rng.randint(0, 40) for _ in seqs])
        elif what == "fork":
            code = h.fork([rng.randrange(6) for _ in seqs], seqs)
        elif what == "free":
            code = h.free(seqs, [rng.randint(0, 20) for _ in seqs])
        else:
            counts = [rng.randint(0, 30) for _ in seqs]
            paths = [sorted(rng.sample(range(max(1, c + rng.randint(0, 1))), min(c, rng.randint(0, 4)))) for c in counts]
            code = h.accept(seqs, counts, 28, paths, 4)
            codes.add(code)
            for (a, x), (b, y) in h.rows_moved:
                assert (a, x) != (b, y)
        if code != OK:
            assert was == (h.refs, h.table, h.len)
        held = [p for row in h.table for p in row if p >= 0]
        assert [held.count(p) for p in range(16)] == h.refs
        for s, m in enumerate(h.len):
            assert [p >= 0 for p in h.table[s]] == [j < h.blocks(m) for j in range(6)]
            if m % 16:
                assert h.refs[h.table[s][m // 16]] == 1
    assert codes == {OK, ESEQ, ELEN, ESHARED, EPATH}


@needs_lib
def test_appended_rows_of_all_heads_are_limited(abi):
    """KV_MAX_HEAD_ROWS counts query and key heads (sizes are looked at before rows: with NULL ones, those that fit are EINVAL)."""
    _abi, lib = abi
    most = _abi.KV_MAX_HEAD_ROWS
    rot = C.byref(rotary(_abi))
    for n, rows, heads, kv in [(64, 32768, 32, 8), (64, 32768, 24, 8), (1, 1 << 20, 32, 32), (1024, 1 << 16, 0, 1),
                               (1024, 1 << 16, 0, 2), (1, 1 << 20, 0, 64), (1, 1 << 20, 1, 64), (1024, 1 << 20, 1024, 1024)]:
        p = C.byref(pages(_abi, n_kv_heads=kv))
        status = lib.kv_pages_append(p, 0, FAKE, n, rows, None, rot, None, heads, None, None, None, None, None)
        assert status == (1 if n * rows * (heads + kv) <= most else 2), (n, rows, heads, kv)
        if status == 2:
            assert b"rows of" in lib.dllm_last_error()


@needs_lib
def test_frequencies_of_their_own_are_one_a_pair(abi):
    """Frequencies in a grid would be read row after row, those of the wrong pairs."""
    import torch

    import paper_2608_11742_amd as P
    f = torch.arange(32, dtype=torch.float32)
    for freq in (f, f.numpy(), f.tolist(), f.double()):
        rot = P.Rotary(64, freq=freq, device="cpu")
        assert rot.freq.tolist() == f.tolist() and rot.freq.dtype == torch.float64 and rot.amplitude == 1.0
    for freq in (f[:31], f[:, None], f[:, None].expand(32, 2), [[x, 0.0] for x in f.tolist()], []):
        with pytest.raises(ValueError):
            P.Rotary(64, freq=freq, device="cpu")
    with pytest.raises(ValueError):
        P.Rotary(64, dim=0, freq=f, device="cpu")
    assert P.Rotary(64, dim=0, device="cpu").dim == 0
