"""Forwards over the paged cache: requests of different lengths and lookahead
branches in one batch, against the oracle's cached forwards."""
import numpy as np
import pytest
import torch

import synth
from synth import ModelShape
from oracle import model as om
from oracle.stats import softmax_stats
from tests.parity import compare_stats, perturbations, allowed_flips

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
SMALL_BF16 = ModelShape(n_layers=2, d_model=512, n_heads=4, head_dim=128, d_ffn=1536, vocab=3000)


@pytest.fixture(scope="module")
def P():
    import paper_2608_11742_amd as P
    return P


def make(P, shape, dtype):
    w_np = synth.model_weights_np(shape, seed=0, dtype=dtype)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    m = P.Model(shape, {k: torch.from_numpy(v).to(DEV).to(td).contiguous() for k, v in w_np.items()}, dtype=dtype,
                max_pos=512)
    return shape, w_np, m


@pytest.fixture(scope="module")
def tiny(P):
    made = make(P, synth.TINY, "f32")
    yield made
    made[2].close()


@pytest.fixture(scope="module")
def small_bf16(P):
    made = make(P, SMALL_BF16, "bf16")
    yield made
    made[2].close()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def toks(tag, n, shape):
    return synth.tokens_np(n + 7, tag, n, shape.vocab - 1)


class Cache:
    """Pages on the GPU and the oracle's (k, v) of the same sequences, per set of weights."""

    def __init__(self, P, model, shape, weights, mirror, page):
        self.P, self.model, self.shape, self.weights, self.mirror = P, model, shape, weights, mirror
        self.kp = model.new_kv_pages(40, page_len=page, max_seqs=10, max_len=256)
        self.kv = [{} for _ in weights]
        self.len = {}
        self.status = ints([0])

    def grow(self, seqs, n):
        self.P.kv_pages_grow(self.kp, ints(seqs), ints([n] * len(seqs)), self.status)
        assert self.status.item() == 0

    def fork(self, src, dst):
        self.P.kv_pages_fork(self.kp, ints([src] * len(dst)), ints(dst), self.status)
        assert self.status.item() == 0
        for kv in self.kv:
            kv.update({d: kv[src] for d in dst})
        self.len.update({d: self.len[src] for d in dst})

    def forward(self, seqs, tokens, lm_pos, **kw):
        """One batch forward (tokens [entries][rows]); returns the statistics and the oracle's logits per weights."""
        n = tokens.shape[1]
        self.grow(seqs, n)
        out = self.model.forward_pages(torch.from_numpy(tokens).to(DEV), self.kp, ints(seqs), ints(lm_pos), **kw)
        torch.cuda.synchronize()
        want = []
        for w, kv in zip(self.weights, self.kv):
            logits, new = [], {}
            for s, t in zip(seqs, tokens):
                own = []
                h = om.hidden(t, w, self.shape, pos_offset=self.len.get(s, 0), mirror=self.mirror,
                              prefix_kv=kv.get(s), collect=own)
                logits.append(om.lm_logits(h[lm_pos], w, self.shape, scale=kw.get("scale", 1.0)))
                new[s] = [(np.concatenate([a[0], b[0]], 1), np.concatenate([a[1], b[1]], 1))
                          for a, b in zip(kv[s], own)] if s in kv else own
            kv.update(new)
            want.append(np.concatenate(logits))
        for s in seqs:
            self.len[s] = self.len.get(s, 0) + n
        return out.numpy(), want


def story(c):
    """Prompts of three requests, branches of the first, then blocks of all of them in one batch, twice."""
    yield c.forward([0], toks("a", 75, c.shape)[None], [3, 74], scale=2.0)
    yield c.forward([1, 2], np.stack([toks("b", 20, c.shape), toks("c", 20, c.shape)]), [0, 19], scale=2.0)
    yield c.forward([2], toks("d", 13, c.shape)[None], [12], scale=2.0)
    c.fork(0, [3, 4, 5])
    block = np.stack([toks(x, 16, c.shape) for x in "efg"])
    block[:, 9:] = c.shape.mask_id
    yield c.forward([3, 4, 5], block, [0, 8, 9, 15], scale=2.0, prefix_seq=0, shared_len=75, max_len=91)
    mixed = np.stack([toks(x, 33, c.shape) for x in "hijk"])
    yield c.forward([1, 4, 2, 0], mixed, [0, 31, 32], scale=2.0)


def test_forward_pages_f32(P, tiny):
    shape, w_np, model = tiny
    for i, (got, want) in enumerate(story(Cache(P, model, shape, [w_np], False, 16))):
        compare_stats(got, softmax_stats(want[0], 16), 1e-4, label=f"forward over pages f32 {i}")


def test_forward_pages_bf16(P, small_bf16):
    shape, w_np, model = small_bf16
    for i, (got, want) in enumerate(story(Cache(P, model, shape, [w_np, *perturbations(w_np)], True, 32))):
        ref, *ref2 = [softmax_stats(x, 16) for x in want]
        compare_stats(got, ref, 2e-2, max_exceptions=allowed_flips(ref, ref2), id_ranks=4,
                      label=f"forward over pages bf16 {i}")


def test_branches_rolled_back_and_tried_again(P, tiny):
    """The same block after kv_pages_free with keep gives the same statistics bit for bit."""
    shape, _, model = tiny
    kp = model.new_kv_pages(20, page_len=16, max_seqs=4, max_len=128)
    st = ints([0])
    P.kv_pages_grow(kp, ints([0]), ints([40]), st)
    model.forward_pages(torch.from_numpy(toks("p", 40, shape))[None].to(DEV), kp, ints([0]), ints([0]))
    P.kv_pages_fork(kp, ints([0, 0]), ints([1, 2]), st)
    block = torch.from_numpy(np.stack([toks("q", 24, shape), toks("r", 24, shape)])).to(DEV)
    seen = []
    for _ in range(3):
        P.kv_pages_grow(kp, ints([1, 2]), ints([24, 24]), st)
        seen.append(model.forward_pages(block, kp, ints([1, 2]), ints([5, 23]), prefix_seq=0, shared_len=40).numpy())
        P.kv_pages_free(kp, ints([1, 2]), st, keep=ints([40, 40]))
        assert st.item() == 0
    assert kp.len.tolist() == [40, 40, 40, 0]
    for s in seen[1:]:
        assert all(np.array_equal(s[k], seen[0][k]) for k in s)


def test_workspace_serves_smaller_forwards(P, tiny):
    shape, _, model = tiny
    kp = model.new_kv_pages(60, page_len=16, max_seqs=8, max_len=128)
    st = ints([0])
    P.kv_pages_grow(kp, ints(list(range(8))), ints([48] * 8), st)
    need = P.dllm_workspace_bytes_pages(model.handle, 8, 48, 48)
    for n, rows, lm in [(1, 1, 1), (8, 48, 48), (3, 17, 5), (8, 2, 2), (1, 48, 48), (5, 33, 1)]:
        assert P.dllm_workspace_bytes_pages(model.handle, n, rows, lm) <= need
        ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)
        out = P.Stats(n * lm, 16, device=DEV)
        t = torch.from_numpy(np.stack([toks(f"w{i}", rows, shape) for i in range(n)])).to(DEV)
        P.dllm_forward_pages(model.handle, t, kp, ints(list(range(n))), ints(list(range(lm))), out, ws)
        assert np.isfinite(out.numpy()["H"]).all()


def test_refusals(P, tiny, small_bf16):
    shape, _, model = tiny
    kp = model.new_kv_pages(10, page_len=16, max_seqs=2, max_len=64)
    t, seqs, lm = torch.zeros(1, 4, dtype=torch.int32, device=DEV), ints([0]), ints([0])
    wrong = [P.KvPages.empty(shape.n_layers + 1, 10, shape.n_heads, 16, shape.head_dim, 2, 4, dtype=torch.float32, device=DEV),
             P.KvPages.empty(shape.n_layers, 10, shape.n_heads * 2, 16, shape.head_dim, 2, 4, dtype=torch.float32, device=DEV),
             P.KvPages.empty(shape.n_layers, 10, shape.n_heads, 16, shape.head_dim, 2, 4, dtype=torch.bfloat16, device=DEV)]
    for kw in [dict(shared_len=-1), dict(prefix_seq=2, shared_len=1), dict(max_len=-1)]:
        with pytest.raises(P.binding.DllmError):
            model.forward_pages(t, kp, seqs, lm, **kw)
    for bad in wrong:
        with pytest.raises(P.binding.DllmError):
            model.forward_pages(t, bad, seqs, lm)
    with pytest.raises(ValueError):
        model.forward_pages(t, kp, ints([0, 1]), lm)
    with pytest.raises(P.binding.DllmError):
        P.dllm_forward_pages(model.handle, t, kp, seqs, lm, P.Stats(1, 16, device=DEV),
                             torch.empty(1024, dtype=torch.uint8, device=DEV))


def test_workspace_alignment(P, tiny):
    shape, _, model = tiny
    kp = model.new_kv_pages(10, page_len=16, max_seqs=2, max_len=64)
    t, seqs, lm = torch.zeros(1, 4, dtype=torch.int32, device=DEV), ints([0]), ints([0])
    ws = torch.empty(P.dllm_workspace_bytes_pages(model.handle, 1, 4, 1) + 16, dtype=torch.uint8, device=DEV)
    for by in (1, 4, 8):
        with pytest.raises(P.binding.DllmError):
            P.dllm_forward_pages(model.handle, t, kp, seqs, lm, P.Stats(1, 16, device=DEV), ws[by:])


def test_forward_captured_and_replayed(P, tiny):
    """Grow, forward and roll back in one graph, one entry of the batch padding;
    every replay bit for bit the eager pass over the same tokens, and as the
    entries by themselves."""
    shape, _, model = tiny
    kp = model.new_kv_pages(30, page_len=16, max_seqs=4, max_len=128)
    st = ints([0])
    P.kv_pages_grow(kp, ints([0]), ints([40]), st)
    model.forward_pages(torch.from_numpy(toks("s", 40, shape))[None].to(DEV), kp, ints([0]), ints([0]))
    P.kv_pages_fork(kp, ints([0, 0]), ints([1, 2]), st)
    seqs, padded, add, keep, lm = ints([1, 2]), ints([1, -1, 2]), ints([24, 24]), ints([40, 40]), ints([5, 23])
    block = torch.zeros(3, 24, dtype=torch.int32, device=DEV)
    out = P.Stats(6, 16, device=DEV)
    ws = torch.empty(P.dllm_workspace_bytes_pages(model.handle, 3, 24, 2), dtype=torch.uint8, device=DEV)

    def step():
        P.kv_pages_grow(kp, seqs, add, st)
        P.dllm_forward_pages(model.handle, block, kp, padded, lm, out, ws, prefix_seq=0, shared_len=40, max_len=64)
        P.kv_pages_free(kp, seqs, st, keep=keep)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(3):
        block.copy_(torch.from_numpy(np.stack([toks(f"{x}{replay}", 24, shape) for x in "tuv"])))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.copy() for k, v in out.numpy().items()}
        assert st.item() == 0 and kp.len.tolist() == [40, 40, 40, 0]
        step()
        torch.cuda.synchronize()
        eager = out.numpy()
        assert all(np.array_equal(eager[k], got[k]) for k in got)
        assert np.isfinite(got["H"]).all()
        for entry, s in ((0, 1), (2, 2)):
            P.kv_pages_grow(kp, ints([s]), ints([24]), st)
            alone = model.forward_pages(block[entry:entry + 1].contiguous(), kp, ints([s]), lm).numpy()
            P.kv_pages_free(kp, ints([s]), st, keep=ints([40]))
            assert np.allclose(alone["H"], got["H"][2 * entry:2 * entry + 2], rtol=1e-4, atol=1e-4)
            assert np.array_equal(alone["argmax"], got["argmax"][2 * entry:2 * entry + 2])
