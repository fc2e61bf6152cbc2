"""Rows of an attention's output that fall on one another are refused on the
host, whatever the strides (runs without a GPU)."""
import ctypes as C
import itertools
import os
import random

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_11742_amd", "libdllm_rps.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libdllm_rps.so not built")

FAKE = 0x10000


@pytest.fixture(scope="module")
def attend():
    """Status of a call with these sizes and strides of out.  Only for rows that overlap: others would be launched."""
    from paper_2608_11742_amd import _abi
    lib = _abi.load()
    p = _abi.KvPagesC(FAKE, FAKE, FAKE, FAKE, FAKE, 2, 10, 1, 64, 16, 4, 8, 1)

    def call(n, rows, heads, seq, row, head, n_rows=None):
        q, out = _abi.Rows(FAKE, 1 << 20, 1 << 10, 64), _abi.Rows(FAKE, seq, row, head)
        ws = lib.kv_pages_attention_workspace_bytes(C.byref(p), n, rows, heads)
        assert ws > 0
        status = lib.kv_pages_attention(C.byref(p), 0, FAKE, n, rows, n_rows, heads, C.byref(q), C.byref(out), 0, 0, 64,
                                        0, 1.0, FAKE, ws, None)
        return status, lib.dllm_last_error()

    return call


def overlap(n, rows, heads, seq, row, head, hd=64):
    at = sorted(b * seq + i * row + h * head for b, i, h in itertools.product(range(n), range(rows), range(heads)))
    return any(y - x < hd for x, y in zip(at, at[1:]))


@pytest.mark.parametrize("n,rows,heads,seq,row,head", [
    (2, 4, 4, 1024, 128, 64),       # heads of a row reach into the next row
    (2, 4, 1, 192, 64, 64),         # rows of an entry reach into the next entry
    (1, 3, 2, 64, 64, 128),         # row 2 of head 0 is row 0 of head 1
    (2, 1, 2, 64, 8, 64),           # entry 1 of head 0 is entry 0 of head 1
    (3, 5, 4, 640, 200, 168),       # only some of them, and in part
    (4, 2, 3, 640, 1984, 64),       # row 1 of entry 0 from inside entry 3 on
    (1024, 64, 1, 4096 - 8, 64, 0),
    (1, 1 << 18, 4, 0, 72, 64),
])
def test_overlapping_rows_are_refused(attend, n, rows, heads, seq, row, head):
    status, text = attend(n, rows, heads, seq, row, head)
    assert status == 2 and b"overlap" in text
    if n * rows * heads < 1 << 17:
        assert overlap(n, rows, heads, seq, row, head)


def test_heads_of_ragged_entries(attend):
    """Which rows n_rows lets be written is known on the device: heads that overlap can be told."""
    for n, rows, heads, seq, row, head in [(2, 4, 4, 1024, 512, 56), (1, 1, 2, 64, 64, 8)]:
        assert attend(n, rows, heads, seq, row, head, FAKE)[0] == 2


def test_random_overlapping_rows_are_refused(attend):
    rng, seen = random.Random(4), 0
    for _ in range(3000):
        n, rows, heads = (rng.randint(1, 5) for _ in range(3))
        strides = [8 * rng.randint(8, 80) for _ in range(3)]
        if overlap(n, rows, heads, *strides):
            status, text = attend(n, rows, heads, *strides)
            assert status == 2 and b"overlap" in text, (n, rows, heads, strides)
            seen += 1
    assert seen > 500
