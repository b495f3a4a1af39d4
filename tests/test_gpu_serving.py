"""The operators of serving from a cache of pages, as they are used together: a
prompt enters in chunks, its tokens' weights add up, the cache is cut down to the
heaviest, and tokens are decoded behind, also from a captured graph.  Attention
and weights are checked against 64 bits at each call (test_gpu_chunk_attention's
bounds, from the values in the cache), what enters the cache against
test_gpu_write_rotated's, the cut against test_gpu_evict's rules."""
import numpy as np
import pytest

import test_gpu_chunk_attention as attention
import test_gpu_evict as evict
import test_gpu_other_streams as streams

pytestmark = pytest.mark.gpu
OK = 0


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_09800_amd import hbf
    hbf.load_library()
    return t


class Server:
    def __init__(self, torch, layers=2, heads=8, kv_heads=2, dim=64, page=16, slots=3, cols=20, dtype="bfloat16", seed=0):
        from paper_2609_09800_amd import hbf
        self.torch, self.layers, self.heads, self.kv_heads, self.dim, self.page = torch, layers, heads, kv_heads, dim, page
        self.dtype, self.dt = dtype, getattr(torch, dtype)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.pool = torch.zeros((layers, 2, 60, page, kv_heads, dim), dtype=self.dt, device="cuda")
        self.tables, self.lens = torch.full((slots, cols), -1, **i32), torch.zeros(slots, **i32)
        self.refs = torch.zeros(60, **i32)
        self.kv = hbf.KvPages(self.pool, refs=self.refs, tables=self.tables, lens=self.lens)
        self.w = torch.zeros((layers, slots, kv_heads, cols * page), device="cuda")
        self.freqs = 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float64, device="cuda") / (dim // 2))
        self.norms = [(1 + 0.2 * torch.randn(dim, generator=self.gen, device="cuda")).to(self.dt) for _ in range(2)]

    def ints(self, a):
        return self.torch.tensor(list(a), dtype=self.torch.int32, device="cuda")

    def qkv(self, n):
        return (2 * self.torch.randn((self.layers, n, self.heads + 2 * self.kv_heads, self.dim), generator=self.gen,
                                     device="cuda")).to(self.dt)

    def layer(self, l, qkv, slots, starts, tok_slots, pos, positions, weights=True, **how):
        """A layer's operators: (q as it was turned, out, lse)."""
        torch, H, K = self.torch, self.heads, self.kv_heads
        q, k, v = qkv[:, :H], qkv[:, H:H + K], qkv[:, H + K:]
        turned, lse = torch.empty((len(qkv), H, self.dim), dtype=self.dt, device="cuda"), torch.empty((len(qkv), H), device="cuda")
        out = torch.empty_like(turned)
        assert self.kv.write_rotated(l, q, k, v, tok_slots, pos, self.freqs, turned, q_weight=self.norms[0],
                                     k_weight=self.norms[1], positions=positions) == OK
        assert self.kv.attention(l, turned, out, slots, starts, lse=lse, weights=self.w[l] if weights else None, **how) == OK
        return turned, out, lse

    def check(self, l, q, out, lse, slots, new, before, window=0, sinks=0):
        b = attention.Batch.__new__(attention.Batch)
        b.torch, b.q, b.pool, b.page, b.dtype = self.torch, q, self.pool[l:l + 1], self.page, self.dtype
        b.slots, b.new, b.tables = np.array(slots), np.array(new), self.tables.cpu().numpy()
        b.starts = np.concatenate([[0], np.cumsum(new)])
        b.lens, b.dev = self.lens.cpu().numpy(), dict(lens=self.lens.cpu())
        b.check(out, lse, b.reference(window=window, sinks=sinks, weights=before), self.w[l])

    def chunk(self, slots, new, positions=None, window=0, sinks=0):
        """New tokens of every row through every layer, checked."""
        lens = self.lens.cpu().numpy()
        assert self.kv.extend(self.ints(slots), self.ints(new)) == OK
        at = [(s, int(lens[s]) + t) for s, n in zip(slots, new) for t in range(n)]
        tok_slots, pos = self.ints(s for s, _ in at), self.ints(p for _, p in at)
        starts = self.ints(np.concatenate([[0], np.cumsum(new)]))
        x = self.qkv(len(at))
        for l in range(self.layers):
            before = self.w[l].clone()
            got = self.layer(l, x[l], self.ints(slots), starts, tok_slots, pos, positions, window=window, sinks=sinks)
            self.check(l, *got, slots, new, before, window, sinks)
        assert self.kv.get_status() == OK

    def cut(self, slots, keep, sinks, recent):
        """Checked against the rules."""
        torch = self.torch
        lens, tables = self.lens.cpu().numpy(), self.tables.cpu().numpy()
        rows = lambda s, n, t: self.pool[:, :, t[s].long().cuda()].flatten(2, 3)[:, :, :n].cpu()
        old = {s: rows(s, int(lens[s]), torch.from_numpy(tables).clamp(min=0)) for s in slots}
        w = self.w.cpu().numpy()
        kept = torch.empty((self.layers, len(slots), self.kv_heads, max(keep)), dtype=torch.int32, device="cuda")
        assert self.kv.evict(self.ints(slots), self.ints(keep), self.w, kept, sinks=sinks, recent=recent) == OK
        assert self.kv.get_status() == OK
        for i, (s, k) in enumerate(zip(slots, keep)):
            end = min(k, int(lens[s]))
            assert int(self.lens[s]) == end
            now = rows(s, end, self.tables.cpu().clamp(min=0))
            for l in range(self.layers):
                for h in range(self.kv_heads):
                    src = evict.choose(w[l, s, h], int(lens[s]), k, sinks, recent)
                    assert kept[l, i, h, :end].tolist() == src
                    assert torch.equal(now[l, :, :, h], old[s][l][:, src, h])
                    assert np.array_equal(self.w[l, s, h, :end].cpu().numpy(), w[l, s, h, src])
                    assert not bool(self.w[l, s, h, end:].any())


@pytest.mark.parametrize("dim,dtype", [(64, "bfloat16"), (128, "float16")])
def test_chunks_weights_cut_and_decode(torch, dim, dtype):
    attention.say(f"serving {dim} {dtype}")
    s = Server(torch, dim=dim, dtype=dtype)
    s.chunk([0, 2], [60, 45])             # two prompts, one of them in a second chunk beside nothing of the other
    s.chunk([0, 2], [70, 0])
    s.cut([2, 0], [30, 64], 4, 12)
    for t in range(4):                    # decoded behind, at the positions that they have in the text
        s.chunk([2, 0], [1, 1], positions=s.ints([45 + t, 130 + t]))
    s.chunk([0, 2, 1], [1, 20, 33])       # one decodes, another goes on with its prompt, a third begins
    s.cut([0, 1, 2], [40, 40, 40], 0, 8)
    s.chunk([0, 1], [1, 1], window=16, sinks=3)
    held = -(-s.lens // s.page)
    assert int((s.refs > 0).sum()) == int(held.sum())


def test_decode_steps_from_a_graph(torch):
    """A step of two layers captured once: the cache grows under it, is cut down between two replays, and grows on."""
    attention.say("serving from a graph")
    s = Server(torch, cols=40)
    s.chunk([0, 1, 2], [50, 10, 31])
    slots, one, starts = s.ints([0, 1, 2]), s.ints([1, 1, 1]), s.ints([0, 1, 2, 3])
    positions, x = s.ints([50, 10, 31]), s.qkv(3)

    def step():
        assert s.kv.extend(slots, one) == OK
        pos = s.lens - 1
        return [s.layer(l, x[l], slots, starts, slots, pos, positions) for l in range(2)]

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        got = step()
    for i in range(20):
        if i == 9:
            s.cut([0, 1, 2], [24, 24, 24], 2, 8)
        x.copy_(s.qkv(3))
        before = s.w.clone()
        g.replay()
        torch.cuda.synchronize()
        for l in range(2):
            s.check(l, *got[l], [0, 1, 2], [1, 1, 1], before[l])
        positions.add_(1)
        assert s.kv.get_status() == OK
    assert s.lens.tolist() == [35, 30, 35]


def test_two_objects_on_two_streams(torch):
    """Two caches at work at the same time: nothing is shared."""
    attention.say("serving on two streams")
    a, b = (attention.Batch(torch, 8, 2, 64, [1, 1, 3], [900, 3000, 70], 16, seed=i) for i in (1, 2))
    want = [x.run() for x in (a, b)]
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = [[torch.empty_like(x.q) for _ in range(30)] for x in (a, b)]
    torch.cuda.synchronize()
    for i in range(30):
        for x, st, o in zip((a, b), s, outs):
            assert x.kv.attention(0, x.q, o[i], x.dev["slots"], x.dev["starts"], stream=st) == OK
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(t, w[0]) for t in o)


@pytest.mark.parametrize("new,lens", [([1, 1], [900, 3000]), ([300, 5], [400, 3000])])
def test_a_busy_stream(torch, new, lens):
    """The call's scratch is known on the stream that it was given."""
    from paper_2609_09800_amd import hbf
    attention.say(f"chunk attention on a busy stream {new}")
    b = attention.Batch(torch, 8, 2, 64, new, lens, 16, seed=3)
    w = b.weights.clone()
    want, _ = b.run(weights=w)
    kv = hbf.KvPages(b.pool, refs=b.dev["refs"], tables=b.dev["tables"], lens=b.dev["lens"])
    out, w2 = torch.full_like(b.q, 7.0), b.weights.clone()
    s = streams.busy(torch)
    assert kv.attention(0, b.q, out, b.dev["slots"], b.dev["starts"], weights=w2, stream=s) == OK
    was = streams.dropped(torch, s, [kv._attn_ws._t, kv._attn_status])
    del kv
    others = streams.others(torch, s, was)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(w, w2)
    assert not any(bool(t.any()) for t in others)
