"""Infinities and numbers that are none in keys and values of the paged cache:
what a sequence does not hold may not reach it."""
import pytest
import torch

from tests.pages_ways import WAYS, ENTRIES, division
from tests.test_gpu_pages import hold, ints, new_pages, poison, queries
from tests.test_gpu_pages_ways import TYPES, batch

pytestmark = pytest.mark.gpu
P = pytest.importorskip("paper_2608_11742_amd")

DEV = "cuda:0"

# entries by themselves, in 16, 32 and 128 rows
ALONE = [
    ("f32", 64, 16, 4, 2, 4, 5, 67, 60, ENTRIES, 0, 16, False, False),
    ("bf16", 64, 32, 2, 2, 4, 6, 96, 40, ENTRIES, 0, 16, False, False),
    ("bf16", 128, 16, 1, 1, 4, 20, 51, 42, ENTRIES, 0, 32, False, False),
    ("bf16", 64, 16, 2, 2, 4, 70, 50, 120, ENTRIES, 0, 128, False, False),
]


def attention(kp, case, seqs, lens, q, counts, causal):
    n, rows, heads = q.shape[:3]
    out = torch.zeros(q.shape, dtype=q.dtype, device=DEV)
    ws = torch.full((P.kv_pages_attention_workspace_bytes(kp, n, rows, heads),), 255, dtype=torch.uint8, device=DEV)
    P.kv_pages_attention(kp, 1, ints(seqs), q, out, ws, n_rows=ints(counts), causal=causal, prefix_seq=0,
                         shared_len=case[7], max_len=max(lens))
    return out


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("what", ["inf", "nan"])
@pytest.mark.parametrize("case", [c for c in WAYS + ALONE if c[5] >= 3 and c[7] >= 2 * c[2] + 4], ids=str)
def test_prefix_past_the_end_of_a_shorter_entry(case, what, causal):
    """Positions of the prefix past the end of the entries that end inside it:
    what they hold may not reach those, however the call is divided."""
    page, n, rows, prefix = case[2], case[5], case[6], case[7]
    kp, seqs, lens = batch(case)
    poison(kp)
    assert division(P.kv_pages_attention_plan(kp, n, rows, case[3], prefix, max(lens))) == case[9:]
    counts = [rows - i % 3 * (rows // 3) for i in range(n)]
    q = queries(n, rows, case[3], case[1], TYPES[case[0]])
    clean = attention(kp, case, seqs, lens, q, counts, causal)
    assert clean.isfinite().all()
    whole = prefix // page * page
    short = lens[2]                                   # the shortest that is not empty
    assert 0 < short < whole
    table, bad = kp.table[0].tolist(), range(short, whole, 5)
    at, slot = (torch.tensor(x, device=DEV) for x in ([table[pos // page] for pos in bad], [pos % page for pos in bad]))
    kp.vt[:, at, :, :, slot] = float("-inf" if what == "inf" else "nan")
    kp.vt[:, at[::2], :, :, slot[::2]] = float("inf" if what == "inf" else "nan")
    if what == "nan":
        kp.k[:, at, :, slot] = float("nan")
    got = attention(kp, case, seqs, lens, q, counts, causal)
    for b in range(n):
        if lens[b] <= short:
            assert torch.equal(got[b], clean[b]), b
        elif not causal:                              # all others see them
            assert not got[b, :counts[b]].isfinite().any(), b


@pytest.mark.parametrize("dtype,rows,lens", [("bf16", 3, [40, 70]), ("bf16", 20, [300, 33]), ("bf16", 140, [500, 200]),
                                             ("f32", 7, [90, 17])])
def test_infinities_that_are_seen(dtype, rows, lens):
    """An infinite value makes its dim infinite, with its sign, in every row of
    the sequence, two of opposite signs make it no number; the other dims and
    the other sequence are as they were."""
    case = (dtype, 64, 16, 2, 2, 2, rows, 0, max(lens))
    kp = hold(new_pages(pages=90, seqs=2, blocks=32, dtype=TYPES[dtype]), lens)
    poison(kp)
    q = queries(2, rows, 2, 64, TYPES[dtype])
    want = attention(kp, case, [0, 1], lens, q, [rows] * 2, False)
    table = kp.table[0].tolist()
    for dim, value, pos in ((3, "inf", lens[0] - 1), (9, "-inf", 5), (20, "inf", lens[0] // 2), (20, "-inf", 0)):
        kp.vt[1, table[pos // 16], :, dim, pos % 16] = float(value)
    got = attention(kp, case, [0, 1], lens, q, [rows] * 2, False)
    want[0, :, :, 3], want[0, :, :, 9], want[0, :, :, 20] = float("inf"), float("-inf"), float("nan")
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(nan=0.0, posinf=1e9, neginf=-1e9), want.nan_to_num(nan=0.0, posinf=1e9, neginf=-1e9))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 5, 40])
def test_write_keeps_what_is_no_number(dtype, rows):
    """Values go in as they are, binary16 saturated for bf16; a NaN stays one."""
    kp = hold(new_pages(pages=20, heads=2, seqs=2, blocks=8, dtype=TYPES[dtype]), [rows + 3, rows + 8])
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.empty(2, rows, 2, 64, dtype=TYPES[dtype], device=DEV).normal_(generator=g) for _ in range(2))
    special = [float("nan"), float("inf"), float("-inf"), 1e6, -1e6, 65504.0, -65504.0, 0.0, 65536.0, 1e-7, -1e-6, -1e-9]
    v[:, :, 0, :12] = torch.tensor(special, device=DEV).to(TYPES[dtype])
    v[0, rows // 2, 1, 5] = k[0, rows // 2, 1, 6] = float("nan")
    P.kv_pages_write(kp, 1, ints([0, 1]), k, v)
    for s, m in enumerate([rows + 3, rows + 8]):
        pos = torch.arange(m - rows, m)
        page, slot = kp.table[s].cpu().long()[pos // 16], pos % 16
        got, keys = kp.vt[1, page.to(DEV), :, :, slot.to(DEV)], kp.k[1, page.to(DEV), :, slot.to(DEV)]
        want = v[s].float().clamp(-65504, 65504).half() if dtype == "bf16" else v[s]
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))
        assert torch.equal(keys.isnan(), k[s].isnan()) and torch.equal(keys.nan_to_num(nan=0.0), k[s].nan_to_num(nan=0.0))


@pytest.mark.parametrize("sizes,strides", [
    ((2, 2, 1), (128, 192, 0)),           # entries and rows between one another, none on another
    ((2, 3, 2), (64, 256, 128)),          # entries innermost
    ((3, 2, 2), (192, 576, 64)),          # heads, entries, rows
    ((2, 5, 2), (320, 64, 640)),          # rows innermost
    ((2, 2, 2), (136, 208, 416)),         # gaps
])
def test_rows_of_any_order_that_do_not_overlap(sizes, strides):
    n, rows, heads = sizes
    kp = hold(new_pages(seqs=3, pages=60, blocks=20, heads=1), [300, 64, 290])
    q = queries(n, rows, heads, 64, torch.bfloat16)
    case = (0,) * 7 + (0,)
    want = attention(kp, case, list(range(n)), [300], q, [rows] * n, False)
    buf = torch.full((4096,), 7.0, dtype=torch.bfloat16, device=DEV)
    out = buf.as_strided((n, rows, heads, 64), (*strides, 1))
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, n, rows, heads), dtype=torch.uint8, device=DEV)
    P.kv_pages_attention(kp, 1, ints(list(range(n))), q, out, ws, max_len=300)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((buf == 7).all())


@pytest.mark.parametrize("hd,rows", [(64, 5), (128, 40)])
def test_ragged_rows_one_after_another(hd, rows):
    """Entries closer to one another than max_rows: their n_rows rows fill the output without a gap."""
    kp = hold(new_pages(seqs=3, pages=60, blocks=20, heads=1, hd=hd), [300, 64, 290])
    q = queries(3, rows, 2, hd, torch.bfloat16)
    counts = [rows // 2] * 3
    want = attention(kp, (0,) * 8, [0, 1, 2], [300], q, counts, True)[:, :rows // 2]
    buf = torch.full((3 * rows * 2 * hd,), 7.0, dtype=torch.bfloat16, device=DEV)
    out = buf.as_strided((3, rows, 2, hd), (rows // 2 * 2 * hd, 2 * hd, hd, 1))
    ws = torch.empty(P.kv_pages_attention_workspace_bytes(kp, 3, rows, 2), dtype=torch.uint8, device=DEV)
    P.kv_pages_attention(kp, 1, ints([0, 1, 2]), q, out, ws, n_rows=ints(counts), causal=True, max_len=300)
    m = want.numel()
    assert torch.equal(buf[:m].view_as(want), want) and bool((buf[m:] == 7).all())
