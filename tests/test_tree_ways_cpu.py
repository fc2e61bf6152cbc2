"""How the attention of drafted trees divides a call, on the host (runs without a GPU)."""
import ctypes as C
import os
import random

import pytest

from tests.pages_ways import ENTRIES, PARTS, PAIRS, division
from tests.test_pages_ways_cpu import pages
from tests.tree_ways import TREE_WAYS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_11742_amd", "libdllm_rps.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libdllm_rps.so not built")


@pytest.fixture(scope="module")
def abi():
    from paper_2608_11742_amd import _abi
    return _abi, _abi.load()


def plan_of(abi, dtype, hd, page, heads, kv, n, rows, shared, most, blocks=1 << 20):
    _abi, lib = abi
    plan = _abi.AttentionPlan()
    p = C.byref(pages(_abi, dtype, hd, page, kv, blocks))
    assert lib.kv_pages_attention_tree_plan(p, n, rows, heads, shared, most, C.byref(plan)) == 0, lib.dllm_last_error()
    return plan, lib.kv_pages_attention_workspace_bytes(p, n, rows, heads)


@pytest.mark.parametrize("case", TREE_WAYS, ids=str)
def test_cases_are_divided_as_they_say(abi, case):
    dtype, hd, page, heads, kv, n, rows, prefix, tail = case[:9]
    plan, _ = plan_of(abi, dtype, hd, page, heads, kv, n, rows, prefix, prefix + tail)
    assert division(plan) == case[9:]


def test_cases_reach_every_launch(abi):
    """Every (type, head_dim, way, rows of the prefix, of the tails, whether the
    tails are of several ranges) of random calls is one of a case, but for
    divided tails behind a prefix of 32 fp32 rows, whose smallest calls are too
    large for a test; and no call's records are more than the workspace holds."""
    have = {(c[0], c[1], *c[9:12], c[13]) for c in TREE_WAYS}
    rng, seen = random.Random(3), set()
    for _ in range(30000):
        dtype, hd, kv = rng.choice(["f32", "bf16"]), rng.choice([64, 128]), rng.choice([1, 2, 3, 4, 8, 16, 32])
        heads = kv * rng.choice([1, 1, 2, 4, 8])
        n, rows = int(2 ** rng.uniform(0, 8)), int(2 ** rng.uniform(0, 9))
        shared = rng.choice([0, int(2 ** rng.uniform(4, 15))])
        most = rng.choice([1, shared, shared + int(2 ** rng.uniform(0, 13)), 1 << 20])
        p, size = plan_of(abi, dtype, hd, rng.choice([16, 64, 256]), heads, kv, n, rows, shared, most)
        seen.add((dtype, hd, p.way, p.prefix_rows, p.tail_rows, p.tail_ranges > 1))
        ranges = p.prefix_ranges + p.tail_ranges
        assert ranges <= 1 or ranges * n * rows * heads * hd * 4 < size
    seen -= {("f32", hd, PARTS, 32, t, True) for hd in (64, 128) for t in (16, 32)}
    assert seen <= have, sorted(seen - have)
    parts = {("bf16", hd, PARTS, p, t) for hd in (64, 128) for p, t in
             [(16, 16), (32, 16), (32, 32), (128, 16), (128, 32), (128, 64), (128, 128)]}
    parts |= {("f32", hd, PARTS, p, t) for hd in (64, 128) for p, t in [(16, 16), (32, 16), (32, 32)]}
    whole = {("f32", hd, ENTRIES, 0, t) for hd in (64, 128) for t in (16, 32)}
    whole |= {("bf16", hd, ENTRIES, 0, t) for hd in (64, 128) for t in (16, 32, 64, 128)}
    pairs = {("bf16", hd, PAIRS, 0, 0) for hd in (64, 128)}
    assert {h[:5] for h in have} == parts | whole | pairs


def test_plan_refusals(abi):
    _abi, lib = abi
    p, plan = pages(_abi, "bf16", 64, 16, 2, 8), _abi.AttentionPlan()

    def ask(n=2, rows=3, heads=4, shared=16, most=64, out=C.byref(plan)):
        return lib.kv_pages_attention_tree_plan(C.byref(p), n, rows, heads, shared, most, out)

    assert ask() == 0 and ask(rows=_abi.KV_TREE_MAX_ROWS) == 0
    assert ask(out=None) == 1 and ask(n=0) == 2 and ask(n=1025) == 2 and ask(heads=3) == 2 and ask(heads=0) == 2
    assert ask(rows=0) == 2 and ask(rows=_abi.KV_TREE_MAX_ROWS + 1) == 2 and b"1024" in lib.dllm_last_error()
    assert ask(shared=-1) == 2 and ask(most=-1) == 2
    p.dtype = 2
    assert ask() == 3


def test_scalings_have_names(abi):
    import paper_2608_11742_amd as P
    with pytest.raises(ValueError):
        P.dllm_rotary_frequencies(64, scaling="log")
    with pytest.raises(P.binding.DllmError):
        P.dllm_rotary_frequencies(-2)


def test_undivided_tails_are_as_long_as_the_call_says(abi):
    """Tails of one range hold the longest sequence there is said to be, in tiles
    of 64, as in the attention without trees, whatever the cache could hold."""
    rng = random.Random(5)
    for _ in range(4000):
        dtype, hd, kv = rng.choice(["f32", "bf16"]), rng.choice([64, 128]), rng.choice([1, 2, 8, 32])
        n, rows, most = int(2 ** rng.uniform(0, 8)), int(2 ** rng.uniform(0, 9)), int(2 ** rng.uniform(0, 17))
        plan, _ = plan_of(abi, dtype, hd, 16, kv * rng.choice([1, 4]), kv, n, rows, 0, most)
        assert plan.way == ENTRIES
        if plan.tail_ranges == 1:
            assert plan.tail_keys == -(-most // 64) * 64
