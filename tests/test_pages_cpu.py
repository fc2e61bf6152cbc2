"""The paged cache's refusals on the host, before any device call, and the host
model the GPU tests compare with (runs without a GPU)."""
import ctypes as C
import os

import numpy as np
import pytest

from tests.pages_model import HostPages, attend, OK, ESEQ, ELEN, ESHARED, EFULL

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_11742_amd", "libdllm_rps.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="libdllm_rps.so not built")

FAKE = 0x10000


@pytest.fixture(scope="module")
def abi():
    from paper_2608_11742_amd import _abi
    return _abi, _abi.load()


def pages(_abi, **kw):
    d = dict(k=FAKE, vt=FAKE, refs=FAKE, table=FAKE, len=FAKE, n_layers=2, n_pages=10, n_kv_heads=2, head_dim=64,
             page_len=16, max_seqs=4, max_blocks=8, dtype=1)
    d.update(kw)
    return _abi.KvPagesC(*[d[f] for f, _ in _abi.KvPagesC._fields_])


BAD_PAGES = [("k", None, 1), ("vt", None, 1), ("refs", None, 1), ("table", None, 1), ("len", None, 1), ("k", FAKE + 8, 1),
             ("dtype", 2, 3), ("head_dim", 96, 2), ("page_len", 8, 2), ("page_len", 48, 2), ("page_len", 512, 2),
             ("n_layers", 0, 2), ("n_pages", 0, 2), ("n_pages", (1 << 20) + 1, 2), ("n_kv_heads", 0, 2),
             ("max_seqs", 0, 2), ("max_seqs", 1025, 2), ("max_blocks", 0, 2), ("max_blocks", (1 << 26) + 1, 2)]


@needs_lib
@pytest.mark.parametrize("field,value,status", BAD_PAGES)
def test_pages_are_checked_by_every_call(abi, field, value, status):
    _abi, lib = abi
    p = C.byref(pages(_abi, **{field: value}))
    r = C.byref(_abi.Rows(FAKE, 64, 64, 64))
    assert lib.kv_pages_init(p, None) == status
    assert lib.kv_pages_grow(p, FAKE, FAKE, 1, FAKE, None) == status
    assert lib.kv_pages_fork(p, FAKE, FAKE, None, 1, FAKE, None) == status
    assert lib.kv_pages_free(p, FAKE, None, 1, FAKE, None) == status
    assert lib.kv_pages_compact(p, FAKE, FAKE, 1 << 30, None) == status
    assert lib.kv_pages_compact_workspace_bytes(p) == 0
    assert lib.kv_pages_write(p, 0, FAKE, 1, 1, None, r, r, None) == status
    assert lib.kv_pages_attention(p, 0, FAKE, 1, 1, None, 2, r, r, 0, 0, 1, 0, 1.0, FAKE, 1 << 40, None) == status
    assert lib.kv_pages_attention_workspace_bytes(p, 1, 1, 2) == 0
    assert lib.dllm_last_error()


@needs_lib
def test_call_arguments(abi):
    _abi, lib = abi
    p = C.byref(pages(_abi))
    for n in (0, -1, 1025):
        assert lib.kv_pages_grow(p, FAKE, FAKE, n, FAKE, None) == 2
        assert lib.kv_pages_fork(p, FAKE, FAKE, None, n, FAKE, None) == 2
        assert lib.kv_pages_free(p, FAKE, None, n, FAKE, None) == 2
    assert lib.kv_pages_grow(p, None, FAKE, 1, FAKE, None) == 1
    assert lib.kv_pages_grow(p, FAKE, None, 1, FAKE, None) == 1
    assert lib.kv_pages_grow(p, FAKE, FAKE, 1, None, None) == 1
    assert lib.kv_pages_fork(p, FAKE, None, None, 1, FAKE, None) == 1
    assert lib.kv_pages_fork(p, FAKE, FAKE, None, 1, None, None) == 1
    assert lib.kv_pages_free(p, FAKE, None, 1, None, None) == 1
    need = lib.kv_pages_compact_workspace_bytes(p)
    assert need > 0
    assert lib.kv_pages_compact(p, FAKE, FAKE, need - 1, None) == 4
    assert lib.kv_pages_compact(p, None, FAKE, need, None) == 1
    assert lib.kv_pages_init(None, None) == 1


@needs_lib
def test_workspace_alignment(abi):
    _abi, lib = abi
    p = C.byref(pages(_abi))
    for ws in (None, FAKE + 1, FAKE + 4, FAKE + 8):
        assert lib.kv_pages_compact(p, FAKE, ws, 1 << 30, None) == 1


@needs_lib
def test_row_arguments(abi):
    _abi, lib = abi
    p = C.byref(pages(_abi))
    good = _abi.Rows(FAKE, 1024, 128, 64)

    def write(k=good, v=good, layer=0, n=1, rows=4):
        return lib.kv_pages_write(p, layer, FAKE, n, rows, None, C.byref(k), C.byref(v), None)

    need = lib.kv_pages_attention_workspace_bytes(p, 2, 4, 4)
    assert need > 0

    def attend_(q=good, o=good, layer=0, n=2, rows=4, heads=4, prefix=0, shared=0, most=64, scale=1.0, ws=FAKE, size=need):
        return lib.kv_pages_attention(p, layer, FAKE, n, rows, None, heads, C.byref(q), C.byref(o), prefix, shared, most,
                                      0, scale, ws, size, None)

    for bad, status in [(_abi.Rows(None, 64, 64, 64), 1), (_abi.Rows(FAKE + 2, 64, 64, 64), 1), (_abi.Rows(FAKE, 64, 60, 64), 1),
                        (_abi.Rows(FAKE, -64, 64, 64), 2), (_abi.Rows(FAKE, 64, 64, (1 << 40) + 8), 2)]:
        assert write(k=bad) == status and write(v=bad) == status
        assert attend_(q=bad) == status and attend_(o=bad) == status
    assert write(layer=2) == 2 and write(layer=-1) == 2 and write(rows=0) == 2 and write(n=0) == 2
    assert write(rows=(1 << 20) + 1) == 2
    assert attend_(layer=2) == 2 and attend_(rows=0) == 2 and attend_(n=0) == 2
    assert attend_(heads=3) == 2 and attend_(heads=0) == 2 and attend_(heads=1026) == 2
    assert attend_(shared=-1) == 2 and attend_(most=-1) == 2
    assert attend_(prefix=4, shared=1) == 1 and attend_(prefix=-1, shared=1) == 1
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert attend_(scale=scale) == 1
    assert attend_(ws=None) == 1 and attend_(ws=FAKE + 4) == 1 and attend_(size=need - 1) == 4
    # rows of the output that fall on one another
    assert attend_(o=_abi.Rows(FAKE, 0, 128, 64)) == 2 and attend_(o=_abi.Rows(FAKE, 1024, 0, 64)) == 2
    assert attend_(o=_abi.Rows(FAKE, 1024, 128, 0)) == 2
    assert lib.kv_pages_attention_workspace_bytes(p, 1024, 1 << 20, 4) == 0


def test_host_model_keeps_its_invariants():
    """References are what the tables hold, no partly filled page is shared, and errors change nothing."""
    import copy
    import random
    rng = random.Random(3)
    h = HostPages(14, 16, 8, 6)
    codes = set()
    for _ in range(400):
        was = copy.deepcopy((h.refs, h.table, h.len))
        what = rng.choice(["grow", "fork", "free", "compact"])
        seqs = [rng.randrange(8) for _ in range(rng.randint(1, 3))]
        if what == "grow":
            code = h.grow(seqs, [rng.randint(0, 40) for _ in seqs])
        elif what == "fork":
            code = h.fork([rng.randrange(8) for _ in seqs], seqs, None if rng.random() < 0.5 else [rng.randint(0, 40) for _ in seqs])
        elif what == "free":
            code = h.free(seqs, None if rng.random() < 0.5 else [rng.randint(0, 40) for _ in seqs])
        else:
            used = h.compact()
            assert all(r > 0 for r in h.refs[:used]) and not any(h.refs[used:])
            code = OK
        codes.add(code)
        if code != OK:
            assert was == (h.refs, h.table, h.len)
        held = [p for row in h.table for p in row if p >= 0]
        assert [held.count(p) for p in range(14)] == h.refs
        for s, m in enumerate(h.len):
            assert [p >= 0 for p in h.table[s]] == [j < h.blocks(m) for j in range(6)]
            if m % 16:
                assert h.refs[h.table[s][m // 16]] == 1
    assert codes == {OK, ESEQ, ELEN, ESHARED, EFULL}


def test_host_attention_is_a_softmax():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(1, 3, 4, 8)), rng.normal(size=(5, 2, 8)), rng.normal(size=(5, 2, 8))
    out, mass, _ = attend(q, [k], [v], [2], True, 0.5)
    assert not out[0, 2].any()
    for i, lim in ((0, 4), (1, 5)):
        for h in range(4):
            w = np.exp(0.5 * k[:lim, h // 2] @ q[0, i, h])
            assert np.allclose(out[0, i, h], (w / w.sum()) @ v[:lim, h // 2])
    assert np.all(mass >= np.abs(out))
    out, _, _ = attend(q, [k[:1]], [v[:1]], [3], True, 0.5)
    assert not out[0, :2].any() and np.allclose(out[0, 2], v[0][[0, 0, 1, 1]])


@needs_lib
def test_forward_pages_without_a_model(abi):
    _abi, lib = abi
    p = C.byref(pages(_abi))
    st = _abi.StatsC(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 16)
    assert lib.dllm_forward_pages(None, FAKE, 1, 4, p, FAKE, 0, 0, 4, FAKE, 1, None, 1.0, None, C.byref(st), FAKE,
                                  1 << 30, None) == 1
    assert lib.dllm_workspace_bytes_pages(None, 1, 4, 1) == 0
