"""The attention over pages on every launch it can take, against 64 bits."""
import pytest
import torch

from tests.pages_ways import WAYS, division
from tests.test_gpu_pages import check_attention, poison, queries, shared_batch

pytestmark = pytest.mark.gpu
P = pytest.importorskip("paper_2608_11742_amd")

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def batch(case):
    """(cache, sequences, lengths): ragged tails, an entry that ends inside the prefix and an empty one where there are several."""
    dtype, hd, page, heads, kv, n, rows, prefix, tail = case[:9]
    own = [tail, tail // 3, -min(prefix, 2 * page + 3), tail - tail // 5, -prefix, 1]
    lens = [max(0, prefix + own[i % len(own)]) for i in range(n)]
    return shared_batch(TYPES[dtype], hd, page, kv, prefix, lens), list(range(1, n + 1)), lens


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("case", WAYS, ids=str)
def test_attention_on_every_launch(case, causal):
    dtype, hd, page, heads, kv, n, rows, prefix, tail = case[:9]
    kp, seqs, lens = batch(case)
    poison(kp)
    assert division(P.kv_pages_attention_plan(kp, n, rows, heads, prefix, max(lens))) == case[9:]
    q = queries(n, rows, heads, hd, TYPES[dtype])
    counts = None if not causal else [max(0, rows - i % 4 * (rows // 3)) for i in range(n)]
    check_attention(kp, 1, seqs, q, counts, causal, prefix_seq=0, shared_len=prefix, max_len=max(lens))
