"""Attention over fp32 pages whose values are near the type's largest: the output
is a mean of them, so it is finite, and as near to 64 bits as that of others."""
import random

import pytest
import torch

import tests.test_gpu_drafts as drafts
from tests.pages_ways import WAYS
from tests.test_gpu_pages import check_attention, hold, new_pages, poison, queries
from tests.test_gpu_pages_ways import batch
from tests.tree_ways import TREE_WAYS

pytestmark = pytest.mark.gpu
P = pytest.importorskip("paper_2608_11742_amd")

F32 = torch.float32


def enlarge(kp):
    """Values of 2^126 .. 2^127, of one sign in a dim, so that nothing cancels."""
    g = torch.Generator(device=kp.device).manual_seed(3)
    kp.vt.uniform_(2.0 ** 126, 2.0 ** 127, generator=g)
    kp.vt[..., 1::2, :] *= -1
    poison(kp)
    return kp


def smallest(cases, key):
    """The smallest fp32 case of each launch."""
    some = sorted((c for c in cases if c[0] == "f32"), key=lambda c: -c[5] * c[6] * c[3] * (c[7] + c[8]))
    return list({key(c): c for c in some}.values())


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", smallest(WAYS, lambda c: (c[1], *c[9:])), ids=str)
def test_attention(case, causal):
    hd, page, heads, kv, n, rows, prefix, tail = case[1:9]
    kp, seqs, lens = batch(case)
    check_attention(enlarge(kp), 1, seqs, queries(n, rows, heads, hd, F32), None, causal, prefix_seq=0, shared_len=prefix,
                    max_len=max(lens))


@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("case", smallest(TREE_WAYS, lambda c: (c[1], *c[9:])), ids=str)
def test_tree_attention(case, kind):
    hd, page, heads, kv, n, rows, prefix, tail = case[1:9]
    kp, seqs, lens = batch(case)
    drafts.check_tree(enlarge(kp), 1, seqs, queries(n, rows, heads, hd, F32), None,
                      drafts.masks(random.Random(n), n, rows, kind), prefix_seq=0, shared_len=prefix, max_len=max(lens))


@pytest.mark.parametrize("equal", [False, True])
@pytest.mark.parametrize("hd,rows,length", [(64, 1, 65536), (128, 5, 70001)])
def test_many_keys(hd, rows, length, equal):
    """A cache that one sequence fills; with equal scores every key weighs the most that one can."""
    kp = enlarge(hold(new_pages(layers=2, pages=-(-length // 256), heads=1, page=256, hd=hd, seqs=1, blocks=-(-length // 256),
                                dtype=F32), [length]))
    q, see = queries(1, rows, 2, hd, F32), drafts.masks(random.Random(1), 1, rows, "tree")
    if equal:
        q = torch.zeros_like(q)
    check_attention(kp, 1, [0], q, None, max_len=length)
    drafts.check_tree(kp, 1, [0], q, None, see, max_len=length)
    # scores that rise to hd, 92 or 185 in log2: the reference moves again and again
    kp.k[1, kp.table[0].long()] = (torch.arange(length + -length % 256, device=kp.device) / length).view(-1, 1, 256, 1).to(F32)
    poison(kp)
    check_attention(kp, 1, [0], torch.ones_like(q), None, scale=1.0, max_len=length)
    drafts.check_tree(kp, 1, [0], torch.ones_like(q), None, see, scale=1.0, max_len=length)


@pytest.mark.parametrize("power", [-80, 126])
@pytest.mark.parametrize("case", smallest(TREE_WAYS, lambda c: (c[1], *c[9:])), ids=str)
def test_powers_of_two(case, power):
    """Values a power of two larger or smaller give outputs that are, bit for bit:
    no weight is rounded otherwise for them and none of the products, of weights
    down to 2^-40 here, leaves the normal numbers."""
    hd, page, heads, kv, n, rows, prefix, tail = case[1:9]
    kp, seqs, lens = batch(case)
    g = torch.Generator(device=kp.device).manual_seed(4)
    kp.vt.uniform_(1.0, 2.0, generator=g)
    kp.vt[..., 1::2, :] *= -1
    q, see = queries(n, rows, heads, hd, F32), drafts.masks(random.Random(n), n, rows, "tree")
    kw = dict(prefix_seq=0, shared_len=prefix, max_len=max(lens))
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, n, rows, heads), dtype=torch.uint8, device=kp.device)

    def both():
        out = torch.empty_like(q)
        P.kv_pages_attention(kp, 1, torch.tensor(seqs, dtype=torch.int32, device=kp.device), q, out, ws, **kw)
        return out, drafts.run_tree(kp, 1, seqs, q, None, see, **kw)

    before = both()
    kp.vt *= 2.0 ** power
    for a, b in zip(before, both()):
        assert bool(torch.isfinite(b).all()) and torch.equal(a.double() * 2.0 ** power, b.double())
