"""What the speed of drafting and verifying over the paged key/value cache is
measured on: queries and keys normed and rotated, rows appended to the cache,
trees of drafted tokens, attention under their masks, accepted rows kept.

listed() names the cases, draw() makes more of the same ranges, prepare()
makes what a program that verifies drafts holds before the call, run() is one
pass through an operator, work() the bytes and operations it cannot do without
and exact() the same outputs in 64 bits.

Kinds of case:
  rotary  queries and keys of a batch normed by head and rotated
  append  the same on the way into the cache: keys and values into the pages
          of one layer, rotated queries out
  tree    parents of drafted tokens into the rows that each sees, and positions
  attend  rows of a tree over the positions before it and their ancestors
  accept  the rows of an accepted path moved to the front of their tree in
          every layer, the rest given back

Where `own` is false, run() computes them in elementary torch operations
(32 bits, angles in 64, rounded once at the end); where it is true, it makes
the library's calls.  Pools: keys [layer][page][head][slot][dim] in the model's
type, values transposed [layer][page][head][dim][slot], binary16 for bf16
models and fp32 for fp32 ones.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"

# heads, key/value heads, head dim
SHAPES = {
    "8b": (32, 32, 128),        # the 8B-class diffusion LLM
    "8b_gqa": (32, 8, 128),     # the same with four query heads to a key head
    "mid": (32, 32, 64),        # generic, 64-wide heads
    "small": (16, 16, 64),      # generic, 64-wide heads
    "tiny": (4, 4, 64),         # the fp32 parity model
}
EPS = 1e-6


# ---------------------------------------------------------------- the cases

def _rotary(**kw):
    return dict(dict(kind="rotary", model="8b_gqa", dtype="bf16", seqs=16, rows=32, first=1000, dim=128,
                     layout="halves", scaling="none", norm=True), **kw)


def _append(**kw):
    return dict(dict(kind="append", model="8b_gqa", dtype="bf16", page=64, seqs=16, rows=32, held_lo=0, held_hi=1024,
                     dim=128, layout="halves", scaling="none", norm=True, tree=False, ragged=False), **kw)


def _tree(**kw):
    return dict(dict(kind="tree", model="tiny", dtype="bf16", page=16, seqs=16, rows=64, held_lo=10, held_hi=300,
                     ragged=False), **kw)


def _attend(**kw):
    return dict(dict(kind="attend", model="8b_gqa", dtype="bf16", page=64, seqs=16, rows=24, shared=0, tail_lo=100,
                     tail_hi=1000, ragged=False), **kw)


def _accept(**kw):
    return dict(dict(kind="accept", model="8b", dtype="bf16", layers=4, page=64, seqs=16, rows=32, path=5, stay=1,
                     held_lo=10, held_hi=1000), **kw)


def listed():
    return [
        # a few rows of an fp32 model with half of each head rotated: nothing but latency
        _rotary(name="rotary_f32_3x7", model="small", dtype="f32", seqs=3, rows=7, dim=32, layout="pairs", norm=False),
        # the prompts of a batch in a scaled long context: 16 x 512 positions
        _rotary(name="rotary_16x512", rows=512, first=90000, scaling="ramp"),
        # one new token of each of 9 sequences
        _append(name="append_9x1", model="small", page=16, seqs=9, rows=1, held_hi=700, dim=64, norm=False),
        # the prompts of a batch into the cache, from odd starts
        _append(name="append_16x512", rows=512),
        # a handful of drafted tokens of one request
        _tree(name="tree_1x5", seqs=1, rows=5),
        # 64 requests with trees of up to 200 tokens
        _tree(name="tree_64x200", seqs=64, rows=200, ragged=True),
        # five drafted tokens of one short request: latency
        _attend(name="attend_1x5_over_150", model="small", page=16, seqs=1, rows=5, tail_lo=150, tail_hi=150),
        # an fp32 model's ragged batch behind an odd shared prefix
        _attend(name="attend_f32_6x13_over_203", model="small", dtype="f32", page=16, seqs=6, rows=13, shared=203,
                tail_lo=14, tail_hi=130, ragged=True),
        # serving: 16 requests behind one instruction, trees of 24 tokens
        _attend(name="attend_16x24_over_1000", shared=1000, tail_lo=40, tail_hi=2500),
        # trees of 64 tokens over four long documents
        _attend(name="attend_4x64_to_60000", page=128, seqs=4, rows=64, tail_lo=20000, tail_hi=60000),
        # short accepted paths of a small fp32 model
        _accept(name="accept_3_small", model="tiny", dtype="f32", layers=2, page=16, seqs=3, rows=9, path=3),
        # 64 requests accept up to 6 of 64 tokens each
        _accept(name="accept_64_of_64", seqs=64, rows=64, path=6, held_hi=500),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "append", "tree", "attend", "attend", "attend", "accept"])
    model = rng.choice(["8b", "8b_gqa", "mid", "small", "tiny"])
    dtype = rng.choice(["bf16", "bf16", "f32"]) if model in ("small", "tiny", "mid") else "bf16"
    page = rng.choice([16, 32, 64, 128])
    hd = SHAPES[model][2]
    turn = dict(dim=rng.choice([hd, hd, hd // 2, hd // 4, 48]), layout=rng.choice(["halves", "pairs"]),
                scaling=rng.choice(["none", "linear", "base", "ramp"]), norm=rng.random() < 0.6)
    if kind == "rotary":
        return _rotary(model=model, dtype=dtype, seqs=_log(rng, 1, 32), rows=_log(rng, 1, 256),
                       first=_log(rng, 1, 1000000), **turn)
    if kind == "append":
        held = _log(rng, 1, 4000)
        return _append(model=model, dtype=dtype, page=page, seqs=_log(rng, 1, 32), rows=_log(rng, 1, 256),
                       held_lo=rng.randint(0, held), held_hi=held, tree=rng.random() < 0.4,
                       ragged=rng.random() < 0.3, **turn)
    if kind == "tree":
        return _tree(page=page, seqs=_log(rng, 1, 64), rows=_log(rng, 1, 200), ragged=rng.random() < 0.4)
    if kind == "accept":
        path = rng.randint(1, 12)
        return _accept(model=model, dtype=dtype, layers=rng.choice([1, 2, 4]), page=page, seqs=_log(rng, 1, 64),
                       path=path, rows=2 * path + _log(rng, 1, 100), stay=rng.randint(0, path),
                       held_lo=rng.randint(0, 100), held_hi=_log(rng, 100, 700))
    seqs, rows = _log(rng, 1, 32), _log(rng, 2, 100)
    shared = rng.choice([0, _log(rng, 1, 8000), _log(rng, 64, 8000)])
    shared = min(shared, 6000000 // (seqs * rows))
    if dtype == "f32":
        shared //= 8
    tail = _log(rng, 1, 1000) if shared else _log(rng, 1, 300000 // (seqs + rows))
    # at most 500 MB of keys and values
    slot = 2 * SHAPES[model][1] * hd * (2 if dtype == "bf16" else 4)
    tail = max(1, min(tail, 500000000 // (slot * seqs) - rows))
    return _attend(model=model, dtype=dtype, page=page, seqs=seqs, rows=rows, shared=shared,
                   tail_lo=rows + rng.randint(0, tail), tail_hi=rows + tail, ragged=rng.random() < 0.3)


# ---------------------------------------------------------------- what the program holds

def _types(dtype):
    return (torch.bfloat16, torch.float16) if dtype == "bf16" else (torch.float32, torch.float32)


def _lengths(n, lo, hi):
    """n lengths from lo to hi, both among them, the longest first."""
    return [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _counts(case):
    """Rows of each sequence: every third one of a ragged batch has fewer."""
    return [case["rows"] - (i % 3) * (case["rows"] // 3) if case.get("ragged") else case["rows"]
            for i in range(case["seqs"])]


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _blocks(positions, page):
    return -(-positions // page)


def _pool(case, layers, pages, g):
    _, hkv, hd = SHAPES[case["model"]]
    tk, tv = _types(case["dtype"])
    k = torch.empty(layers, pages, hkv, case["page"], hd, dtype=tk, device=DEV).normal_(generator=g)
    vt = torch.empty(layers, pages, hkv, hd, case["page"], dtype=tv, device=DEV).normal_(generator=g)
    return k, vt


def _meta(s, pages, blocks, lists, lens):
    """References, tables and lengths in one buffer; lists: the pages of each sequence."""
    seqs = len(lens)
    meta = torch.zeros(pages + seqs * blocks + seqs, dtype=torch.int32)
    refs, table, length = meta[:pages], meta[pages:pages + seqs * blocks].view(seqs, blocks), meta[-seqs:]
    table.fill_(-1)
    for i, (held, m) in enumerate(zip(lists, lens)):
        at = torch.tensor(held, dtype=torch.int64)
        table[i, :len(held)] = at.int()
        refs.index_add_(0, at, torch.ones(len(held), dtype=torch.int32))
        length[i] = m
    s.meta = meta.to(DEV)
    s.refs, s.table, s.len = (s.meta[:pages], s.meta[pages:pages + seqs * blocks].view(seqs, blocks),
                              s.meta[-seqs:])


def _parents(rng, rows):
    """A tree of drafts in the order they were made; now and then another root."""
    return [-1 if i == 0 or rng.random() < 0.02 else rng.randint((i - 1) // 4, (i - 1) // 2) for i in range(rows)]


def _see(parents):
    """Rows that each row sees, as the bits of a whole number."""
    bits = []
    for i, p in enumerate(parents):
        bits.append(1 << i | (bits[p] if p >= 0 else 0))
    return bits


def _words(bits, words):
    """A whole number as signed 32-bit words, the lowest first."""
    w = [bits >> 32 * j & 0xffffffff for j in range(words)]
    return [x - (1 << 32) if x >> 31 else x for x in w]


def _turn(case, g):
    """Frequencies and factor of a case's rotation, by the definition of its scaling, and gains."""
    hd, dim = SHAPES[case["model"]][2], case["dim"]
    base, factor, length, slow, fast = 10000.0, 8.0, 4096.0, 1.0, 32.0
    amplitude = 1.0
    if case["scaling"] == "base" and dim > 2:
        base *= factor ** (dim / (dim - 2))
    freq = [base ** (-2 * j / dim) for j in range(dim // 2)]
    if case["scaling"] == "linear":
        freq = [f / factor for f in freq]
    elif case["scaling"] == "ramp":
        amplitude = 0.1 * math.log(factor) + 1.0
        part = [min(1.0, max(0.0, (length * f / (2 * math.pi) - slow) / (fast - slow))) for f in freq]
        freq = [f * (p + (1 - p) / factor) for f, p in zip(freq, part)]
    t = SimpleNamespace(dim=dim, layout=case["layout"], norm=case["norm"], amplitude=amplitude, factor=factor,
                        length=length, slow=slow, fast=fast, q_gain=None, k_gain=None)
    t.freq = torch.tensor(freq, dtype=torch.float64, device=DEV)
    if t.norm:
        t.q_gain = 1 + 0.2 * torch.empty(hd, device=DEV).normal_(generator=g)
        t.k_gain = 1 + 0.2 * torch.empty(hd, device=DEV).normal_(generator=g)
    return t


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    hq, hkv, hd = SHAPES[case["model"]]
    tk, _ = _types(case["dtype"])
    n, rows, kind = case["seqs"], case["rows"], case["kind"]
    s = SimpleNamespace(case=case, counts=_counts(case))
    s.n_rows = _ints(s.counts) if case.get("ragged") else None
    if kind in ("rotary", "append", "attend"):
        # a [row][q k v] projection
        qkv = torch.empty(n, rows, hq + 2 * hkv, hd, dtype=tk, device=DEV).normal_(generator=g)
        s.q, s.new_k, s.new_v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
        s.out = torch.zeros(n, rows, hq, hd, dtype=tk, device=DEV)
    if kind in ("rotary", "append"):
        s.turn = _turn(case, g)
    if kind == "rotary":
        s.k_out = torch.zeros(n, rows, hkv, hd, dtype=tk, device=DEV)
        s.pos = _ints([[case["first"] + rng.randint(0, case["first"] // 8) + i for i in range(rows)] for _ in range(n)])
        return s
    page = case["page"]
    if kind == "attend":
        # sequence 0 is the prefix; whole pages of it are shared, the cut one is each one's own
        shared = case["shared"]
        whole = shared // page
        lens = [shared] + [shared + t for t in _lengths(n, case["tail_lo"], case["tail_hi"])]
        need = [_blocks(m, page) - whole for m in lens[1:]]
        pages = _blocks(shared, page) + sum(need) + 3
        free = iter(rng.sample(range(pages), pages))
        first = [next(free) for _ in range(_blocks(shared, page))]
        lists = [first] + [first[:whole] + [next(free) for _ in range(m)] for m in need]
        s.k, s.vt = _pool(case, 2, pages, g)
        _meta(s, pages, _blocks(max(lens), page), lists, lens)
        s.seqs = _ints(range(1, n + 1))
        s.max_len = max(lens)
    else:
        lens = [m + rows for m in _lengths(n, case["held_lo"], case["held_hi"])]
        need = [_blocks(m, page) for m in lens]
        free = iter(rng.sample(range(sum(need) + 2), sum(need) + 2))
        _meta(s, sum(need) + 2, max(need), [[next(free) for _ in range(m)] for m in need], lens)
        layers = 1 if kind == "tree" else 2 if kind == "append" else case["layers"]
        s.k, s.vt = _pool(case, layers, sum(need) + 2, g)
        s.seqs = _ints(rng.sample(range(n), n))
    s.layer = 1
    if kind in ("tree", "attend") or case.get("tree"):
        s.parents = [_parents(rng, rows) for _ in range(n)]
        s.words = (rows + 31) // 32
        s.see = [_see(p) for p in s.parents]
    if kind == "tree":
        s.parent = _ints(s.parents)
        s.mask = torch.zeros(n, rows, s.words, dtype=torch.int32, device=DEV)
        s.pos = torch.zeros(n, rows, dtype=torch.int32, device=DEV)
    elif kind == "attend":
        s.mask = _ints([[_words(bits, s.words) for bits in see] for see in s.see])
    elif kind == "append":
        s.pos = None
        if case["tree"]:    # positions by depth, in call order of the sequences
            at = s.seqs.tolist()
            s.pos = _ints([[lens[at[b]] - s.counts[b] + bin(bits).count("1") - 1 for bits in s.see[b]]
                           for b in range(n)])
    elif kind == "accept":
        # the first rows of a path where they are, the others from behind every place that is filled
        stay = min(case["stay"], case["path"])
        s.paths = []
        for b in range(n):
            m = max(stay, case["path"] - b % 3)
            s.paths.append(list(range(stay)) + sorted(rng.sample(range(m, rows), m - stay)))
        s.path = _ints([p + [0] * (case["path"] - len(p)) for p in s.paths])
        s.n_path = _ints([len(p) for p in s.paths])
        s.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        s.saved = s.meta.clone()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2608_11742_amd as P
        s.P = P
        if case["kind"] in ("rotary", "append"):
            t = s.turn
            s.rot = P.Rotary(SHAPES[case["model"]][2], dim=t.dim, layout=t.layout, base=10000.0,
                             scaling=None if case["scaling"] == "none" else case["scaling"], factor=t.factor,
                             original_len=t.length, slow=t.slow, fast=t.fast, norm=t.norm, eps=EPS, q_gain=t.q_gain,
                             k_gain=t.k_gain, device=DEV)
        if case["kind"] != "rotary":
            s.pages = P.KvPages(s.k, s.vt, s.refs, s.table, s.len)
        if case["kind"] == "attend":
            need = P.kv_pages_attention_workspace_bytes(s.pages, s.q.shape[0], s.q.shape[1], s.q.shape[2])
            s.ws = torch.empty(need, dtype=torch.uint8, device=DEV)
        elif case["kind"] == "accept":
            need = P.kv_pages_accept_workspace_bytes(s.pages, case["seqs"], case["path"])
            s.ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return {"rotary": _run_rotary, "append": _run_append, "tree": _run_tree, "attend": _run_attend,
            "accept": _run_accept}[s.case["kind"]](s)


def _rotated(t, x, pos, gain):
    """x [n][rows][heads][hd] normed and rotated to positions pos [n][rows], in 32 bits."""
    y = x.float()
    if t.norm:
        y = y / torch.sqrt((y * y).mean(3, keepdim=True) + EPS) * gain
    if t.dim == 0:
        return y
    angle = (pos.double()[:, :, None] * t.freq)[:, :, None]
    c, s = (torch.cos(angle) * t.amplitude).float(), (torch.sin(angle) * t.amplitude).float()
    half = t.dim // 2
    a, b = (y[..., :half], y[..., half:t.dim]) if t.layout == "halves" else (y[..., 0:t.dim:2], y[..., 1:t.dim:2])
    a, b = a * c - b * s, a * s + b * c
    turned = torch.cat([a, b], 3) if t.layout == "halves" else torch.stack([a, b], 4).flatten(3)
    return torch.cat([turned, y[..., t.dim:]], 3)


def _run_rotary(s):
    if own:
        s.P.rotary_rows(s.rot, s.q, s.out, s.new_k, s.k_out, pos=s.pos)
        return [s.out, s.k_out]
    return [_rotated(s.turn, s.q, s.pos, s.turn.q_gain).to(s.q.dtype),
            _rotated(s.turn, s.new_k, s.pos, s.turn.k_gain).to(s.q.dtype)]


def _rows_of(s):
    """First position [n], rows [n] and which rows there are [n][rows], on the device."""
    n, rows = s.case["seqs"], s.case["rows"]
    count = torch.full((n,), rows, dtype=torch.int64, device=DEV) if s.n_rows is None else s.n_rows.long()
    i = torch.arange(rows, device=DEV)[None]
    return s.len[s.seqs.long()].long() - count, count, i < count[:, None]


def _run_append(s):
    if own:
        s.P.kv_pages_append(s.pages, s.layer, s.seqs, s.new_k, s.new_v, s.rot, q=s.q, q_out=s.out, pos=s.pos,
                            n_rows=s.n_rows)
        return [s.k[s.layer], s.vt[s.layer], s.out]
    page = s.case["page"]
    first, _, there = _rows_of(s)
    at = first[:, None] + torch.arange(s.case["rows"], device=DEV)[None]
    pos = at if s.pos is None else s.pos
    q = _rotated(s.turn, s.q, pos, s.turn.q_gain).to(s.q.dtype)
    k = _rotated(s.turn, s.new_k, pos, s.turn.k_gain).to(s.q.dtype)
    v = s.new_v.float()
    v = (v.clamp(-65504, 65504) if s.vt.dtype == torch.float16 else v).to(s.vt.dtype)
    column = (at // page).clamp(max=s.table.shape[1] - 1)
    where, slot = s.table[s.seqs.long()].long().gather(1, column)[there], (at % page)[there]
    s.k[s.layer][where, :, slot] = k[there]
    s.vt[s.layer][where, :, :, slot] = v[there]
    s.out[there] = q[there]
    return [s.k[s.layer], s.vt[s.layer], s.out]


def _run_tree(s):
    if own:
        s.P.kv_pages_tree(s.pages, s.seqs, s.parent, s.mask, s.pos, n_rows=s.n_rows)
        return [s.mask, s.pos]
    n, rows = s.parent.shape
    first, _, there = _rows_of(s)
    i = torch.arange(rows, device=DEV)
    # a row reaches itself and its parent; squared, the ancestors twice as far
    reach = ((s.parent[:, :, None] == i) | (i[:, None] == i)).float()
    steps = 1
    while steps < rows:
        reach = (torch.matmul(reach, reach) > 0).float()
        steps *= 2
    bits = torch.zeros(n, rows, 32 * s.words, dtype=torch.int64, device=DEV)
    bits[:, :, :rows] = reach.long()
    word = (bits.view(n, rows, s.words, 32) << torch.arange(32, device=DEV)).sum(3)
    word = torch.where(word >= 1 << 31, word - (1 << 32), word).int()
    s.mask.copy_(torch.where(there[:, :, None], word, s.mask))
    s.pos.copy_(torch.where(there, (first[:, None] + reach.sum(2).long() - 1).int(), s.pos))
    return [s.mask, s.pos]


def _run_attend(s):
    c = s.case
    if own:
        s.P.kv_pages_attention_tree(s.pages, s.layer, s.seqs, s.q, s.out, s.mask, s.ws, n_rows=s.n_rows, prefix_seq=0,
                                    shared_len=c["shared"], max_len=s.max_len)
        return s.out
    n, rows, hq, hd = s.q.shape
    hkv = s.k.shape[2]
    group = hq // hkv
    at = s.table[s.seqs.long()].clamp(min=0).long()
    keys = s.k[s.layer][at].float().permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, hd)
    values = s.vt[s.layer][at].float().permute(0, 2, 1, 4, 3).reshape(n, hkv, -1, hd)
    q = s.q.float().reshape(n, rows, hkv, group, hd).permute(0, 2, 1, 3, 4).reshape(n, hkv, rows * group, hd)
    scores = torch.matmul(q, keys.transpose(2, 3).contiguous()) / math.sqrt(hd)
    first, count, there = _rows_of(s)
    # column by column: before the tree, or a row of it that the mask names
    bits = (s.mask[:, :, :, None] >> torch.arange(32, device=DEV) & 1).flatten(2)[:, :, :rows] > 0
    column = torch.arange(scores.shape[3], device=DEV)[None] - first[:, None]
    inside = (column >= 0) & (column < count[:, None])
    named = bits.gather(2, column.clamp(0, rows - 1)[:, None].expand(n, rows, -1))
    seen = (column < 0)[:, None] | inside[:, None] & named
    scores = scores.masked_fill(~seen.repeat_interleave(group, 1)[:, None], -math.inf)
    top = scores.amax(3, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    e = torch.exp(scores - top)
    o = torch.matmul(e, values) / e.sum(3, keepdim=True).clamp(min=torch.finfo(torch.float32).tiny)
    o = o.reshape(n, hkv, rows, group, hd).permute(0, 2, 1, 3, 4).reshape(n, rows, hq, hd)
    return torch.where(there[:, :, None, None], o.to(s.out.dtype), s.out)


def _run_accept(s):
    # the tables before the acceptance again; the rows that move are still where they were
    s.meta.copy_(s.saved)
    if own:
        s.P.kv_pages_accept(s.pages, s.seqs, s.path, s.n_path, s.status, s.ws, rows=s.case["rows"])
        return [s.k, s.vt, s.refs, s.table, s.len, s.status]
    page, at = s.case["page"], s.seqs.long()
    first, _, _ = _rows_of(s)
    j = torch.arange(s.path.shape[1], device=DEV)[None]
    moved = (j < s.n_path[:, None]) & (s.path != j)
    source, target = first[:, None] + s.path.long(), first[:, None] + j
    last = s.table.shape[1] - 1
    table = s.table[at].long()
    p0, s0 = table.gather(1, (source // page).clamp(max=last))[moved], (source % page)[moved]
    p1, s1 = table.gather(1, (target // page).clamp(max=last))[moved], (target % page)[moved]
    s.k[:, p1, :, s1] = s.k[:, p0, :, s0]
    s.vt[:, p1, :, :, s1] = s.vt[:, p0, :, :, s0]
    length = first + s.n_path.long()
    drop = (torch.arange(last + 1, device=DEV)[None] >= ((length + page - 1) // page)[:, None]) & (table >= 0)
    s.refs.index_add_(0, table.clamp(min=0).reshape(-1), -drop.int().reshape(-1))
    s.table[at] = torch.where(drop, -1, table).int()
    s.len[at] = length.int()
    return [s.k, s.vt, s.refs, s.table, s.len, s.status]


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    hq, hkv, hd = SHAPES[case["model"]]
    size = 2 if case["dtype"] == "bf16" else 4
    counts, rows, page = _counts(case), case["rows"], case.get("page", 1)
    slot = 2 * hkv * hd * size                   # key and value of one position in one layer
    if case["kind"] == "rotary":
        return {"bytes": 2 * sum(counts) * (hq + hkv) * hd * size + 4 * sum(counts), "flops": 0}
    if case["kind"] == "append":
        return {"bytes": 2 * sum(counts) * (hq + 2 * hkv) * hd * size, "flops": 0}
    if case["kind"] == "tree":
        return {"bytes": sum(counts) * 4 * (2 + (rows + 31) // 32), "flops": 0}
    if case["kind"] == "accept":
        stay = min(case["stay"], case["path"])
        moved = sum(max(stay, case["path"] - b % 3) - stay for b in range(case["seqs"]))
        return {"bytes": 2 * moved * case["layers"] * slot + 4 * case["seqs"] * (case["path"] + 1), "flops": 0}
    shared = case["shared"]
    tails = _lengths(case["seqs"], case["tail_lo"], case["tail_hi"])
    whole = shared // page * page                # the positions that all read from the same pages
    positions = whole + sum(shared - whole + t for t in tails)
    # a row sees what is before the tree and, of a tree like these, some log2 of it
    seen = sum(m * (shared + t - m + max(1, m.bit_length() - 1)) for t, m in zip(tails, counts))
    return {"bytes": positions * slot + 2 * sum(counts) * hq * hd * size + 4 * (positions // page),
            "flops": 4 * seen * hq * hd}


# ---------------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    return {"rotary": _exact_rotary, "append": _exact_append, "tree": _exact_tree, "attend": _exact_attend,
            "accept": _exact_accept}[case["kind"]](s)


def _exact_turn(t, x, pos, gain):
    """One pair of elements at a time as a complex number, all rows and heads at once."""
    y = x.double()
    if t.norm:
        y = y * torch.rsqrt(y.pow(2).sum(3, keepdim=True) / y.shape[3] + EPS) * gain.double()
    out = y.clone()
    for j, f in enumerate(t.freq.tolist()):
        a, b = (j, j + t.dim // 2) if t.layout == "halves" else (2 * j, 2 * j + 1)
        w = torch.polar(torch.full(pos.shape, t.amplitude, dtype=torch.float64, device=DEV), pos.double() * f)
        z = torch.complex(y[..., a], y[..., b]) * w[:, :, None]
        out[..., a], out[..., b] = z.real, z.imag
    return out


def _exact_rotary(s):
    return [_exact_turn(s.turn, s.q, s.pos, s.turn.q_gain), _exact_turn(s.turn, s.new_k, s.pos, s.turn.k_gain)]


def _exact_append(s):
    k, vt, out = s.k[s.layer].double(), s.vt[s.layer].double(), s.out.double()
    lens, table, page = s.len.tolist(), s.table.tolist(), s.case["page"]
    for b, seq in enumerate(s.seqs.tolist()):
        m, first = s.counts[b], lens[seq] - s.counts[b]
        pos = torch.arange(first, first + m, device=DEV)[None] if s.pos is None else s.pos[b:b + 1, :m]
        out[b, :m] = _exact_turn(s.turn, s.q[b:b + 1, :m], pos, s.turn.q_gain)[0]
        new = _exact_turn(s.turn, s.new_k[b:b + 1, :m], pos, s.turn.k_gain)[0]
        for j in range(first // page, (lens[seq] - 1) // page + 1):
            lo, hi = max(first, j * page), min(lens[seq], (j + 1) * page)
            p, at = table[seq][j], slice(lo - j * page, hi - j * page)
            k[p][:, at] = new[lo - first:hi - first].permute(1, 0, 2)
            v = s.new_v[b, lo - first:hi - first].double().permute(1, 2, 0)
            vt[p][:, :, at] = v.clamp(-65504, 65504) if s.vt.dtype == torch.float16 else v
    return [k, vt, out]


def _exact_tree(s):
    lens, rows = s.len.tolist(), s.case["rows"]
    mask, pos = [], []
    for b, seq in enumerate(s.seqs.tolist()):
        m, first = s.counts[b], lens[seq] - s.counts[b]
        mask.append([_words(bits, s.words) for bits in s.see[b][:m]] + [[0] * s.words] * (rows - m))
        pos.append([first + bin(bits).count("1") - 1 for bits in s.see[b][:m]] + [0] * (rows - m))
    return [_ints(mask), _ints(pos)]


def _exact_attend(s):
    """Sequence by sequence and head by head: softmax over the positions before the tree and the row's ancestors."""
    n, rows, hq, hd = s.q.shape
    hkv = s.k.shape[2]
    if sum(s.len.tolist()) * rows * hq > 2_000_000_000:
        return None
    lens, table = s.len.tolist(), s.table.tolist()
    out = s.out.double()
    for b in range(n):
        m, c = lens[b + 1], s.counts[b]
        held = torch.tensor([p for p in table[b + 1] if p >= 0], device=DEV)
        keys, values = s.k[s.layer][held], s.vt[s.layer][held]
        hidden = torch.tensor([[not bits >> j & 1 for j in range(c)] for bits in s.see[b][:c]])
        hidden = torch.cat([torch.zeros(c, m - c, dtype=torch.bool), hidden], 1).to(DEV)
        for h in range(hq):
            kv = h * hkv // hq
            kh = torch.cat(list(keys[:, kv].double().unbind(0)), 0)[:m]
            vh = torch.cat(list(values[:, kv].double().unbind(0)), 1)[:, :m]
            z = torch.mm(s.q[b, :c, h].double(), kh.t().contiguous()) * hd ** -0.5
            z[hidden] = -math.inf
            out[b, :c, h] = torch.mm(torch.softmax(z, 1), vh.t().contiguous())
    return out


def _exact_accept(s):
    """One row after the other, on the host's tables."""
    refs, table, lens = s.refs.tolist(), s.table.tolist(), s.len.tolist()
    page, rows = s.case["page"], s.case["rows"]
    k, vt = s.k.double(), s.vt.double()
    for b, seq in enumerate(s.seqs.tolist()):
        first = lens[seq] - rows
        for j, r in enumerate(s.paths[b]):
            (a, x), (c, y) = divmod(first + r, page), divmod(first + j, page)
            k[:, table[seq][c], :, y] = s.k[:, table[seq][a], :, x].double()
            vt[:, table[seq][c], :, :, y] = s.vt[:, table[seq][a], :, :, x].double()
        lens[seq] = first + len(s.paths[b])
        for c in range(_blocks(lens[seq], page), len(table[seq])):
            if table[seq][c] >= 0:
                refs[table[seq][c]] -= 1
                table[seq][c] = -1
    return [k, vt, _ints(refs), _ints(table), _ints(lens), s.status]
