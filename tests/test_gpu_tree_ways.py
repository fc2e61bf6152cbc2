"""The attention of drafted trees on every launch it can take, over uneven
lengths and what is sent for `max_len`, and the tensors of its calls."""
import random

import pytest
import torch

import tests.test_gpu_drafts as drafts
from tests.pages_ways import division
from tests.test_gpu_pages import hold, ints, new_pages, poison, queries
from tests.test_gpu_pages_ways import TYPES, batch
from tests.tree_ways import TREE_WAYS

pytestmark = pytest.mark.gpu
P = pytest.importorskip("paper_2608_11742_amd")

DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("case", TREE_WAYS, ids=str)
def test_every_launch(case):
    """Trees, or masks of any pattern over fewer rows in some entries."""
    dtype, hd, page, heads, kv, n, rows, prefix, tail = case[:9]
    kp, seqs, lens = batch(case)
    poison(kp)
    kw = dict(prefix_seq=0, shared_len=prefix, max_len=max(lens))
    assert division(P.kv_pages_attention_tree_plan(kp, n, rows, heads, prefix, max(lens))) == case[9:]
    kind = "any" if n > 1 and (rows + tail) % 2 else "tree"
    counts = None if kind == "tree" else [max(0, rows - i % 4 * max(1, rows // 3)) for i in range(n)]
    drafts.check_tree(kp, 1, seqs, queries(n, rows, heads, hd, TYPES[dtype]), counts,
                      drafts.masks(random.Random(n), n, rows, kind), **kw)


# the smallest of each launch, where rows see a first row that others do not
SMALLEST = sorted((c for c in TREE_WAYS if c[6] > 1), key=lambda c: -c[5] * c[6] * c[3] * (c[7] + c[8]))
WILD = list({(c[0], c[1], *c[9:12], c[13]): c for c in SMALLEST}.values())


@pytest.mark.parametrize("what", ["inf", "nan", "lowest"])
@pytest.mark.parametrize("case", WILD, ids=str)
def test_values_that_a_row_does_not_see(case, what):
    drafts.test_values_that_a_row_does_not_see(case, what)


@pytest.mark.parametrize("dtype,hd,heads,kv,rows,longest", [
    (BF16, 64, 2, 2, 5, 3000), (BF16, 128, 4, 1, 6, 3000), (BF16, 128, 4, 4, 40, 2500), (BF16, 64, 4, 1, 30, 4000),
    (F32, 64, 2, 2, 9, 2000), (F32, 128, 4, 2, 40, 1500),
])
@pytest.mark.parametrize("kind", ["one", "two", "equal", "none", "steps"])
def test_uneven_lengths(dtype, hd, heads, kv, rows, longest, kind):
    """One long sequence among short and empty ones, equal lengths, none at all; `max_len` right, too small and too large."""
    lens = {"one": [0, 1, longest, 0, rows, 63], "two": [longest, longest // 2] + [rows] * 9, "equal": [longest // 3] * 7,
            "none": [0, 0, 0], "steps": [rows + 64 * i for i in range(20)]}[kind]
    n, page = len(lens), 32
    kp = hold(new_pages(pages=2 + sum(-(-m // page) for m in lens), heads=kv, page=page, hd=hd, seqs=n,
                        blocks=max(1, -(-max(lens) // page)), dtype=dtype), lens)
    poison(kp)
    q, see = queries(n, rows, heads, hd, dtype), drafts.masks(random.Random(n), n, rows, "tree")
    for most in (max(lens), 1, None):
        drafts.check_tree(kp, 0, list(range(n)), q, None, see, max_len=most)


@pytest.mark.parametrize("n", [1, 63, 64, 65, 200])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_entries(n, dtype):
    lens = [(37 * i) % 700 for i in range(n)]
    lens[n // 2] = 2000
    kp = hold(new_pages(pages=2 + sum(-(-m // 16) for m in lens), heads=1, page=16, hd=64, seqs=n, blocks=125, dtype=dtype), lens)
    poison(kp)
    for rows in (3, 34):
        q, see = queries(n, rows, 2, 64, dtype), drafts.masks(random.Random(n), n, rows, "tree")
        drafts.check_tree(kp, 1, list(range(n))[::-1], q, None, see, max_len=2000)


def test_two_streams_and_named_ones():
    """Two calls at once, on streams that are named or current, each with a workspace of its own."""
    kp = hold(new_pages(seqs=3, pages=90, blocks=40, heads=2), [600, 33, 410])
    q = [queries(3, rows, 4, 64, BF16) for rows in (7, 40)]
    see = [drafts.masks(random.Random(rows), 3, rows, "tree") for rows in (7, 40)]
    want = [drafts.run_tree(kp, 1, [0, 1, 2], x, None, s) for x, s in zip(q, see)]
    masks = [drafts.bits_of(s, x.shape[1]) for x, s in zip(q, see)]
    ws = [torch.full((P.kv_pages_attention_workspace_bytes(kp, 3, x.shape[1], 4),), 255, dtype=torch.uint8, device=DEV) for x in q]
    out = [torch.zeros_like(x) for x in q]
    seqs, streams = ints([0, 1, 2]), [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        P.kv_pages_attention_tree(kp, 1, seqs, q[0], out[0], masks[0], ws[0], stream=streams[0])
        with torch.cuda.stream(streams[1]):
            P.kv_pages_attention_tree(kp, 1, seqs, q[1], out[1], masks[1], ws[1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    rot, pos = P.Rotary(64, device=DEV), ints([[5] * 7] * 3)
    a, b = torch.zeros_like(q[0]), torch.zeros_like(q[0])
    P.rotary_rows(rot, q[0], a, pos=pos)
    torch.cuda.synchronize()
    P.rotary_rows(rot, q[0], b, pos=pos, stream=streams[0].cuda_stream)
    streams[0].synchronize()
    assert torch.equal(a, b)


def test_arguments_of_other_kinds():
    kp = hold(new_pages(seqs=3), [40, 20, 0])
    rot, q = P.Rotary(64, device=DEV), queries(2, 3, 2, 64, BF16)
    out, two, mask = torch.empty_like(q), ints([0, 1]), torch.zeros(2, 3, 1, dtype=torch.int32, device=DEV)
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, 2, 3, 2), dtype=torch.uint8, device=DEV)
    attend = lambda **kw: P.kv_pages_attention_tree(kp, kw.pop("layer", 0), kw.pop("seqs", two), kw.pop("q", q), out,
                                                    kw.pop("mask", mask), kw.pop("ws", ws), **kw)
    for call in (lambda: attend(seqs=[0, 1]), lambda: attend(mask=None), lambda: attend(q=3), lambda: attend(ws=None),
                 lambda: attend(ws="ws"), lambda: attend(q=q.expand(2, 3, 2, 64)[0]), lambda: P.rotary_rows(rot, [1.0], out),
                 lambda: P.rotary_rows(rot, q[:, :1].expand(2, 3, 2, 64), out, n_rows=7),
                 lambda: P.rotary_rows(rot, q[:, :, :1].expand(2, 3, (1 << 32) + 1, 64), out)):
        with pytest.raises((ValueError, P.binding.DllmError)):
            call()
    for call in (lambda: attend(max_len=1 << 40), lambda: attend(layer=1 << 33), lambda: attend(shared_len=-(1 << 35))):
        with pytest.raises(OverflowError):
            call()
    for call in (lambda: attend(layer=1.5), lambda: attend(scale="1"), lambda: attend(max_len="long")):
        with pytest.raises(TypeError):
            call()
    for scale in (1e60, float("nan")):
        with pytest.raises(P.binding.DllmError):
            attend(scale=scale)
