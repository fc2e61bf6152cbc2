"""How the attention over pages divides a call, on the host (runs without a GPU)."""
import ctypes as C
import itertools
import os
import random

import pytest

from tests.pages_ways import WAYS, ENTRIES, PARTS, PAIRS, division

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2608_11742_amd", "libdllm_rps.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libdllm_rps.so not built")

FAKE = 0x10000


@pytest.fixture(scope="module")
def abi():
    from paper_2608_11742_amd import _abi
    return _abi, _abi.load()


def pages(_abi, dtype, hd, page, kv, blocks):
    return _abi.KvPagesC(FAKE, FAKE, FAKE, FAKE, FAKE, 1, 1 << 20, kv, hd, page, 1024, blocks, int(dtype == "bf16"))


def plan_of(abi, dtype, hd, page, heads, kv, n, rows, shared, most, blocks=1 << 20):
    _abi, lib = abi
    plan = _abi.AttentionPlan()
    status = lib.kv_pages_attention_plan(C.byref(pages(_abi, dtype, hd, page, kv, blocks)), n, rows, heads, shared,
                                         most, C.byref(plan))
    assert status == 0, lib.dllm_last_error()
    return plan


@pytest.mark.parametrize("case", WAYS, ids=str)
def test_cases_are_divided_as_they_say(abi, case):
    dtype, hd, page, heads, kv, n, rows, prefix, tail = case[:9]
    plan = plan_of(abi, dtype, hd, page, heads, kv, n, rows, prefix, prefix + tail)
    assert division(plan) == case[9:]
    if plan.way == PARTS:
        assert plan.prefix_ranges * plan.prefix_keys >= prefix // page * page
    if plan.way != PAIRS:
        assert plan.tail_keys % 64 == 0 and plan.tail_ranges >= 1


def test_cases_reach_every_launch(abi):
    """Every (type, head_dim, way, rows of the prefix, of the tails) that
    random calls take is one that a case has (entries by themselves in bf16
    and in 16 rows are the cases of the plain attention tests)."""
    have = {(c[0], c[1], *c[9:12]) for c in WAYS}
    rng = random.Random(2)
    seen = set()
    for _ in range(30000):
        dtype, hd, kv = rng.choice(["f32", "bf16"]), rng.choice([64, 128]), rng.choice([1, 2, 3, 4, 8, 16, 32])
        heads = kv * rng.choice([1, 1, 2, 4, 8])
        n, rows = int(2 ** rng.uniform(0, 8)), int(2 ** rng.uniform(0, 7))
        shared = int(2 ** rng.uniform(4, 15))
        most = rng.choice([1, shared, shared + int(2 ** rng.uniform(0, 11)), 1 << 20])
        p = plan_of(abi, dtype, hd, rng.choice([16, 64, 256]), heads, kv, n, rows, shared, most)
        if p.way != ENTRIES or (dtype == "f32" and p.tail_rows == 32):
            seen.add((dtype, hd, p.way, p.prefix_rows, p.tail_rows))
    assert seen <= have, sorted(seen - have)
    parts = {("f32", hd, PARTS, p, t) for hd in (64, 128) for p, t in [(16, 16), (32, 16), (32, 32)]}
    parts |= {("bf16", hd, PARTS, p, t) for hd in (64, 128)
              for p, t in itertools.product((16, 32, 128), repeat=2) if p >= t}
    pairs = {("bf16", hd, PAIRS, 0, 0) for hd in (64, 128)}
    whole = {("f32", hd, ENTRIES, 0, 32) for hd in (64, 128)}
    assert have == parts | pairs | whole


def test_plan_refusals(abi):
    _abi, lib = abi
    p, plan = pages(_abi, "bf16", 64, 16, 2, 8), _abi.AttentionPlan()

    def ask(n=2, rows=3, heads=4, shared=16, most=64, out=C.byref(plan)):
        return lib.kv_pages_attention_plan(C.byref(p), n, rows, heads, shared, most, out)

    assert ask() == 0
    assert ask(out=None) == 1
    assert ask(n=0) == 2 and ask(n=1025) == 2 and ask(rows=0) == 2 and ask(heads=3) == 2
    assert ask(shared=-1) == 2 and ask(most=-1) == 2
    assert lib.kv_pages_attention_plan(None, 2, 3, 4, 16, 64, C.byref(plan)) == 1


def test_limits_of_the_header(abi):
    """Every KV_MAX_ number of the header is the binding's, and is the last value that is taken."""
    import re
    _abi, lib = abi
    text = open(os.path.join(ROOT, "include", "dllm_rps.h")).read()
    limits = {k: eval(v) for k, v in re.findall(r"#define (KV_MAX_\w+) +([()\d <]+\d\)?)", text)}
    assert len(limits) == 7
    for name, value in limits.items():
        assert getattr(_abi, name) == value, name

    def ask(n=1, rows=1, heads=1, kv=1, **kw):
        p = pages(_abi, "bf16", 64, 16, kv, 8)
        for field, value in kw.items():
            setattr(p, field, value)
        return lib.kv_pages_attention_plan(C.byref(p), n, rows, heads, 0, 64, C.byref(_abi.AttentionPlan()))

    for kw in [dict(n=1024), dict(rows=1 << 20), dict(heads=1024), dict(heads=1024, kv=1024), dict(n_pages=1 << 20),
               dict(max_seqs=1024), dict(n_layers=65536), dict(max_blocks=1 << 26), dict(n=64, rows=1 << 20),
               dict(n=1024, rows=64, heads=1024)]:
        assert ask(**kw) == 0, kw
        name, value = list(kw.items())[-1]
        over = {**kw, name: value + 1}
        assert ask(**over) == 2, over
