"""Rotations, appended rows and acceptances of the largest sizes, and caches
past 2^32 bytes."""
import random

import pytest
import torch

import tests.test_gpu_drafts as drafts
from tests.test_gpu_pages import hold, ints, queries

pytestmark = pytest.mark.gpu
P = pytest.importorskip("paper_2608_11742_amd")

DEV = "cuda:0"
BF16 = torch.bfloat16


def test_as_many_rows_as_there_may_be():
    """2^26 rows of one head, rotated and appended: the same as some of them by themselves."""
    n, rows, hd = 64, 1 << 20, 64
    x = torch.empty(n, rows, 1, hd, dtype=BF16, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    rot = P.Rotary(hd, device=DEV)
    out = torch.zeros_like(x)
    P.rotary_rows(rot, x, out)
    page = 256
    kp = P.KvPages.empty(1, n * rows // page, 1, page, hd, n, rows // page, dtype=BF16, device=DEV)
    st, seqs = ints([9]), torch.arange(n, dtype=torch.int32, device=DEV)
    P.kv_pages_grow(kp, seqs, torch.full((n,), rows, dtype=torch.int32, device=DEV), st)
    P.kv_pages_append(kp, 0, seqs, x, x, rot)
    assert st.item() == 0
    for b, at in [(0, 0), (0, 777216), (1, 4096), (31, 524288), (n - 1, rows - page)]:
        want = torch.zeros(1, page, 1, hd, dtype=BF16, device=DEV)
        P.rotary_rows(rot, x[b:b + 1, at:at + page], want, pos_offset=at)
        assert torch.equal(out[b, at:at + page], want[0])
        held = kp.table[b, at // page].item()
        assert torch.equal(kp.k[0, held, 0], want[0, :, 0])
        assert torch.equal(kp.vt[0, held, 0].t(), x[b, at:at + page, 0].half())
    blocks = out.view(n, -1, page * hd)
    assert bool((blocks.view(torch.int16).abs().amax(-1) > 0).all())


def test_an_acceptance_of_many_layers():
    """1024 entries over 2^18 layers and heads: the one row that moves, moves in all of them."""
    layers, heads, hd, page = 4096, 64, 64, 16
    kp = P.KvPages.empty(layers, 2, heads, page, hd, 1024, 2, dtype=BF16, device=DEV)
    kp.k.normal_()
    kp.vt.normal_()
    st, seqs = ints([9]), torch.arange(1024, dtype=torch.int32, device=DEV).flip(0).contiguous()
    P.kv_pages_grow(kp, ints([5]), ints([20]), st)
    k, vt = kp.k.clone(), kp.vt.clone()
    a, b = kp.table[5].tolist()
    rows, path, n_path = (torch.zeros(1024, dtype=torch.int32, device=DEV) for _ in range(3))
    rows[1018], path[1018], n_path[1018] = 7, 6, 1
    ws = torch.empty(P.kv_pages_accept_workspace_bytes(kp, 1024, 1), dtype=torch.uint8, device=DEV)
    P.kv_pages_accept(kp, seqs, path[:, None], n_path, st, ws, rows=8, n_rows=rows)
    assert st.item() == 0 and kp.len[5].item() == 14 and kp.table[5].tolist() == [a, -1]
    k[:, a, :, 13], vt[:, a, :, :, 13] = k[:, b, :, 3], vt[:, b, :, :, 3]
    assert torch.equal(kp.k, k) and torch.equal(kp.vt, vt)


@pytest.mark.parametrize("rows", [3, 40])
def test_pages_past_32_bits(rows):
    """A round over the last pages of 10 GB of keys: as over the same pages in a small cache."""
    pages, heads, page, hd, lens = 20000, 8, 256, 128, [600, 90, 1000]
    big = P.KvPages.empty(1, pages, heads, page, hd, 3, 8, dtype=BF16, device=DEV)
    small = hold(P.KvPages.empty(1, 12, heads, page, hd, 3, 8, dtype=BF16, device=DEV), lens)
    small.k.normal_(generator=torch.Generator(device=DEV).manual_seed(3))
    small.vt.normal_(generator=torch.Generator(device=DEV).manual_seed(4))
    big.k[0, pages - 12:] = small.k[0]
    big.vt[0, pages - 12:] = small.vt[0]
    big.table.copy_(torch.where(small.table >= 0, small.table + pages - 12, small.table))
    big.refs[pages - 12:] = small.refs
    big.len.copy_(small.len)
    rng, seqs, rot = random.Random(1), ints([2, 0, 1]), P.Rotary(hd, device=DEV)
    see = drafts.masks(rng, 3, rows, "tree")
    q, k, v = (queries(3, rows, h, hd, BF16) for h in (16, heads, heads))
    outs, st = [], ints([9])
    for kp in (small, big):
        q_out = torch.zeros_like(q)
        P.kv_pages_append(kp, 0, seqs, k, v, rot, q=q, q_out=q_out)
        outs.append(drafts.run_tree(kp, 0, [2, 0, 1], q_out, None, see))
        ws = torch.empty(P.kv_pages_accept_workspace_bytes(kp, 3, 2), dtype=torch.uint8, device=DEV)
        P.kv_pages_accept(kp, seqs, ints([[1, 2], [0, 2], [2, 0]]), ints([2, 2, 1]), st, ws, rows=rows)
        assert st.item() == 0
    assert torch.equal(*outs)
    assert torch.equal(big.k[0, pages - 12:], small.k[0]) and torch.equal(big.vt[0, pages - 12:], small.vt[0])
    assert torch.equal(big.len, small.len) and torch.equal((big.table + 1).clamp(min=0) > 0, (small.table + 1) > 0)
