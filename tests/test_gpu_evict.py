"""Sequences cut down by their tokens' weights, against a sequential model of the
same rules: every table, count, length, kept place, weight and byte of the pool
must be equal."""
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

OK, EINVAL = 0, -1


def say(msg):
    print(f"[gpu-case] {msg}", flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_09800_amd import hbf
    hbf.load_library()
    return t


def choose(weights, L, keep, sinks, recent):
    """The old position of the token at each place."""
    if keep >= L:
        return list(range(L))
    m = keep - recent
    w = np.where(np.isnan(weights[:L]), -np.inf, weights[:L])
    nan = np.isnan(weights[:L])
    order = sorted(range(sinks, L - recent), key=lambda p: (nan[p], -w[p], p))
    best = sorted(order[:m - sinks])
    movers = [p for p in best if p >= m]
    stay = set(p for p in best if p < m)
    src = list(range(sinks))
    for p in range(sinks, m):
        src.append(p if p in stay else movers.pop(0))
    assert not movers
    return src + list(range(L - recent, L))


class Cache:
    def __init__(self, torch, layers, heads, dim, page, lens, seed=0, cols=1, share=(), wide=0):
        from paper_2609_09800_amd import hbf
        self.torch, self.page = torch, page
        rng = np.random.default_rng(seed)
        n = len(lens) + 1
        held = np.array([-(-x // page) for x in lens] + [0])
        pages = int(held.sum()) + 3
        perm = rng.permutation(pages).astype(np.int32)
        self.tables = np.full((n, int(held.max()) + cols), -1, np.int32)
        self.refs = np.zeros(pages, np.int32)
        self.lens = np.array(list(lens) + [0], np.int32)
        at = 0
        for s in range(n):
            self.tables[s, :held[s]] = perm[at:at + held[s]]
            at += held[s]
        for s, col, to in share:   # the same page in another row too
            self.tables[to, col] = self.tables[s, col]
        for s in range(n):
            for p in self.tables[s, :held[s]]:
                self.refs[p] += 1
        self.pool = rng.integers(-30000, 30000, (layers, 2, pages, page, heads, dim)).astype(np.int16)
        w = np.exp(rng.standard_normal((layers, n, heads, self.tables.shape[1] * page + wide)) * 2).astype(np.float32)
        w[rng.random(w.shape) < 0.2] = 0.0
        self.weights = w
        c = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.dev = dict(tables=c(self.tables), refs=c(self.refs), lens=c(self.lens), pool=c(self.pool), weights=c(w))
        self.kv = hbf.KvPages(self.dev["pool"].view(torch.bfloat16), refs=self.dev["refs"], tables=self.dev["tables"],
                              lens=self.dev["lens"])

    def ints(self, a):
        return self.torch.from_numpy(np.array(a, np.int32)).cuda()

    def evict(self, slots, keep, sinks=0, recent=0, max_keep=None, out=False):
        torch = self.torch
        layers, heads = self.pool.shape[0], self.pool.shape[4]
        max_keep = max(keep, default=0) if max_keep is None else max_keep
        kept = torch.full((layers, len(slots), heads, max_keep), -7, dtype=torch.int32, device="cuda")
        w_out = torch.full_like(self.dev["weights"], 7.0) if out else None
        assert self.kv.evict(self.ints(slots), self.ints(keep), self.dev["weights"], kept, sinks=sinks, recent=recent,
                             weights_out=w_out) == OK
        return kept, w_out

    def model(self, slots, keep, sinks, recent, max_keep, out=False):
        layers, heads = self.pool.shape[0], self.pool.shape[4]
        kept = np.full((layers, len(slots), heads, max_keep), -1, np.int32)
        w_out = np.full_like(self.weights, 7.0) if out else self.weights
        for i, (s, k) in enumerate(zip(slots, keep)):
            L = int(self.lens[s])
            end = min(L, k)
            place = lambda j: (self.tables[s, j // self.page], j % self.page)
            old = {j: self.pool[:, :, place(j)[0], place(j)[1]].copy() for j in range(L)}
            old_w = self.weights[:, s].copy()
            for l in range(layers):
                for h in range(heads):
                    src = choose(old_w[l, h], L, k, sinks, recent)
                    kept[l, i, h, :end] = src
                    for j, p in enumerate(src):
                        self.pool[l, :, place(j)[0], place(j)[1], h] = old[p][l, :, h]
                    w_out[l, s, h, :end] = old_w[l, h, src]
                    w_out[l, s, h, end:L] = 0.0
            for c in range(-(-end // self.page), -(-L // self.page)):
                self.refs[self.tables[s, c]] -= 1
                self.tables[s, c] = -1
            self.lens[s] = end
        return kept, w_out

    def both(self, slots, keep, sinks=0, recent=0, max_keep=None, out=False):
        max_keep = max(keep, default=0) if max_keep is None else max_keep
        kept, w_out = self.evict(slots, keep, sinks, recent, max_keep, out)
        want, want_w = self.model(slots, keep, sinks, recent, max_keep, out)
        assert self.kv.get_status() == OK
        assert np.array_equal(kept.cpu().numpy(), want)
        got_w = (w_out if out else self.dev["weights"]).cpu().numpy()
        assert np.array_equal(got_w, want_w, equal_nan=True)
        self.same()

    def same(self):
        for name in ("tables", "refs", "lens", "pool"):
            equal = np.array_equal(self.dev[name].cpu().numpy(), getattr(self, name))
            assert equal, name
        assert np.array_equal(self.dev["weights"].cpu().numpy(), self.weights, equal_nan=True)


CASES = [
    # layers, heads, dim, page, lengths, keep, sinks, recent
    (1, 1, 64, 16, [1], [1], 0, 0),
    (1, 1, 64, 16, [1], [0], 0, 0),
    (1, 2, 64, 16, [2, 40], [1, 0], 0, 0),
    (2, 2, 128, 16, [33, 100], [32, 50], 4, 8),
    (2, 3, 64, 24, [130, 7, 300], [20, 7, 299], 0, 0),
    (1, 4, 128, 1, [37, 64], [12, 30], 3, 9),
    (3, 1, 64, 7, [200, 500, 13], [100, 64, 64], 1, 60),
    (1, 2, 64, 16, [400], [64], 32, 32),            # nothing between the first and the last
    (1, 2, 64, 16, [400], [100], 100, 0),
    (1, 2, 64, 16, [400], [100], 0, 100),
    (1, 1, 64, 16, [1200], [1199], 0, 700),         # the last ones move over themselves
    (1, 1, 64, 256, [1500, 900], [700, 890], 5, 400),
    (1, 1, 64, 16, [12000], [5000], 4, 10),         # more free places than are listed at a time
    (1, 1, 64, 64, [20000], [9800], 0, 0),
]


@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_against_the_model(torch, case, out):
    layers, heads, dim, page, lens, keep, sinks, recent = case
    say(f"evict {case} {out}")
    c = Cache(torch, layers, heads, dim, page, lens, seed=sum(lens))
    order = np.random.default_rng(1).permutation(len(lens))
    c.both([int(i) for i in order], [keep[i] for i in order], sinks, recent, out=out)


@pytest.mark.parametrize("out", [False, True])
@pytest.mark.parametrize("L", [60, 6000])
def test_weights_of_any_value(torch, out, L):
    """Ties, both zeros, negative ones, infinities and NaN (the lowest): equal ones go by position."""
    for seed in range(4):
        say(f"evict values {L} {out} {seed}")
        c = Cache(torch, 1, 2, 64, 16, [L, L - 7], seed=seed)
        rng = np.random.default_rng(seed)
        some = np.array([0.0, -0.0, 1.0, -1.0, np.inf, -np.inf, np.nan, 1e-45, -1e-45, 3e38], np.float32)
        c.weights[:] = some[rng.integers(0, [10, 4, 2, 7][seed], c.weights.shape)]
        c.dev["weights"].copy_(torch.from_numpy(c.weights))
        c.both([1, 0], [L // 3, L // 2], 2, 5, out=out)


def test_all_weights_equal_keeps_the_first(torch):
    c = Cache(torch, 1, 1, 64, 16, [5000], seed=1)
    c.weights[:] = 0.0
    c.dev["weights"].zero_()
    kept, _ = c.evict([0], [100], 3, 10)
    assert kept[0, 0, 0].tolist() == list(range(90)) + list(range(4990, 5000))


@pytest.mark.parametrize("keep", [20, 45])
def test_shared_pages(torch, keep):
    """Pages that other rows hold: read, kept as they are before the first written place, and given up."""
    c = Cache(torch, 2, 2, 64, 8, [90, 24, 90], seed=2, share=[(0, 0, 1), (0, 1, 1), (0, 11, 2)])
    # (share replaces entries of rows 1 and 2 by pages of row 0; both hold them now)
    c.both([0], [keep], sinks=16, recent=2)


@pytest.mark.parametrize("what", ["slot", "slot_low", "twice", "keep", "keep_low", "cut", "len", "len_low", "weights",
                                  "shared", "page", "page_low", "free"])
def test_refused_with_nothing_changed(torch, what):
    say(f"evict refused {what}")
    share = [(0, 3, 1)] if what == "shared" else []
    c = Cache(torch, 2, 2, 64, 16, [100, 120, 90], seed=3, share=share)
    slots, keep, max_keep = [0, 2], [70, 60], None
    if what.startswith("slot"):
        slots = [0, -1 if what == "slot_low" else 4]
    elif what == "twice":
        slots = [2, 2]
    elif what == "keep":
        max_keep = 69
    elif what == "keep_low":
        keep = [70, -1]
    elif what == "cut":
        keep = [70, 9]         # fewer than the first and the last that stay
    elif what.startswith("len"):
        c.lens[2] = -1 if what == "len_low" else c.tables.shape[1] * 16 + 1
        c.dev["lens"].copy_(torch.from_numpy(c.lens))
    elif what == "weights":
        c.weights = c.weights[..., :99].copy()
        c.dev["weights"] = torch.from_numpy(c.weights).cuda()
    elif what.startswith("page"):
        c.tables[2, 4] = -1 if what == "page_low" else len(c.refs)
        c.dev["tables"].copy_(torch.from_numpy(c.tables))
    elif what == "free":
        c.refs[c.tables[2, 5]] = 0
        c.dev["refs"].copy_(torch.from_numpy(c.refs))
    kept, w_out = c.evict(slots, keep, 4, 6, max_keep=max_keep, out=True)
    assert c.kv.get_status() == EINVAL and c.kv.get_status() == OK
    assert bool((w_out == 7.0).all())
    c.same()


def test_list_of_every_slot_and_of_none(torch):
    lens = [(i * 37) % 90 for i in range(300)]
    c = Cache(torch, 1, 1, 64, 8, lens, seed=4)
    c.both(list(range(300)), [30] * 300, 2, 8)
    c.both([], [], 0, 0)
    c.both([300], [0], 5, 5)   # an empty row is not cut


def test_weights_inside_a_wider_tensor(torch):
    c = Cache(torch, 2, 3, 64, 16, [100, 50], seed=5, wide=9)
    wide = torch.full((2, 3, 3, c.weights.shape[-1] + 4), 5.0, device="cuda")
    wide[..., :-4] = c.dev["weights"]
    c.dev["weights"] = wide[..., :-4]
    c.both([1, 0], [20, 64], 1, 3)
    assert bool((wide[..., -4:] == 5.0).all())


def test_host_refusals(torch):
    from paper_2609_09800_amd import hbf
    c = Cache(torch, 2, 2, 64, 16, [100, 50], seed=6)
    w, s, k = c.dev["weights"], c.ints([0]), c.ints([40])
    kept = torch.empty((2, 1, 2, 40), dtype=torch.int32, device="cuda")
    for args, how in (((s.long(), k, w, kept), {}), ((s, c.ints([40, 41]), w, kept), {}), ((s, k, w.double(), kept), {}),
                      ((s, k, w[:1], kept), {}), ((s, k, w[:, :1], kept), {}), ((s, k, w[:, :, :1], kept), {}),
                      ((s, k, w[..., ::2], kept), {}), ((s, k, w[:1].expand(2, -1, -1, -1), kept), {}),
                      ((s, k, w, kept[:1]), {}), ((s, k, w, kept.float()), {}), ((s.cpu(), k, w, kept), {}),
                      ((s, k, w, kept), dict(weights_out=w[..., :-1])), ((s, k, w, kept), dict(weights_out=w.cpu()))):
        with pytest.raises(hbf.HbfError):
            c.kv.evict(*args, **how)
    for how in (dict(sinks=-1), dict(recent=-1)):
        assert c.kv.evict(s, k, w, kept, **how) == EINVAL
    assert c.kv.get_status() == OK
    c.same()


def test_several_in_turn_with_extend_and_fork(torch):
    """The cache goes on after a cut: pages come back, rows grow, are cut again and shared."""
    c = Cache(torch, 1, 2, 64, 16, [300, 200], seed=7, cols=6)
    for turn in range(4):
        say(f"evict turn {turn}")
        keep = [120 - 10 * turn, 90]
        c.both([0, 1], keep, 4, 16)
        assert int((c.dev["refs"] > 0).sum()) == sum(-(-int(x) // 16) for x in c.lens)
        assert c.kv.extend(c.ints([0, 1]), c.ints([50, 33])) == OK and c.kv.get_status() == OK
        c.tables, c.refs, c.lens = (c.dev[n].cpu().numpy().copy() for n in ("tables", "refs", "lens"))
        assert c.lens.tolist() == [keep[0] + 50, 123, 0]
    assert c.kv.fork(c.ints([0]), c.ints([2])) == OK and c.kv.get_status() == OK
    # (a fork copies the last page, which both will write)
    c.tables, c.refs, c.lens, c.pool = (c.dev[n].cpu().numpy().copy() for n in ("tables", "refs", "lens", "pool"))
    kept, _ = c.evict([0], [80], 4, 16)      # would write into shared pages
    assert c.kv.get_status() == EINVAL
    c.same()
    c.both([0], [100], 100, 0)               # nothing is written


def test_another_stream_and_graph(torch):
    c, d = (Cache(torch, 2, 2, 64, 16, [300, 200, 77], seed=8) for _ in range(2))
    w0, t0, r0, l0, p0 = (c.dev[n].clone() for n in ("weights", "tables", "refs", "lens", "pool"))
    s = torch.cuda.Stream()
    slots, keep = c.ints([2, 0]), c.ints([50, 128])
    kept = torch.empty((2, 2, 2, 128), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert c.kv.evict(slots, keep, c.dev["weights"], kept, sinks=4, recent=20, stream=s) == OK
    s.synchronize()
    want, _ = d.evict([2, 0], [50, 128], 4, 20)
    assert torch.equal(kept, want) and torch.equal(c.dev["pool"], d.dev["pool"])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert c.kv.evict(slots, keep, c.dev["weights"], kept, sinks=4, recent=20) == OK
    for i in range(4):
        for n, v in (("weights", w0 if i % 2 else w0.flip(-1)), ("tables", t0), ("refs", r0), ("lens", l0), ("pool", p0)):
            c.dev[n].copy_(v)
            d.dev[n].copy_(v)
        keep.copy_(c.ints([50 - i, 128 - 20 * i]))
        g.replay()
        torch.cuda.synchronize()
        want, _ = d.evict([2, 0], [50 - i, 128 - 20 * i], 4, 20, max_keep=128)
        assert torch.equal(kept, want)
        for n in ("weights", "tables", "refs", "lens", "pool"):
            assert torch.equal(c.dev[n], d.dev[n]), n
        assert c.kv.get_status() == OK


def test_largest_lists(torch):
    """65,535 slots of one layer; and more choices a launch than the moves have workgroups for."""
    for slots, heads, layers, L, keep, recent in ((65535, 1, 1, 3, 2, 1), (600, 16, 4, 40, 24, 8)):
        say(f"evict largest {slots} {heads} {layers}")
        from paper_2609_09800_amd import hbf
        i32 = dict(dtype=torch.int32, device="cuda")
        held = -(-L // 8)
        gen = torch.Generator(device="cuda").manual_seed(9)
        pool = torch.randn((layers, 2, slots * held, 8, heads, 64), generator=gen, device="cuda").bfloat16()
        tables, lens = torch.arange(slots * held, **i32).view(slots, held).flip(0).contiguous(), torch.full((slots,), L, **i32)
        old, was = pool.clone(), tables.clone()
        kv = hbf.KvPages(pool, refs=torch.ones(slots * held, **i32), tables=tables, lens=lens)
        w = torch.rand((layers, slots, heads, L), generator=gen, device="cuda")
        w0 = w.clone()
        kept = torch.empty((layers, slots, heads, keep), **i32)
        assert kv.evict(torch.arange(slots, **i32), torch.full((slots,), keep, **i32), w, kept, recent=recent) == OK
        assert kv.get_status() == OK and bool((lens == keep).all())
        # the heaviest of those before the last ones, which stay the last
        m = keep - recent
        best = w0[..., :L - recent].topk(m, -1).indices.sort(-1).values
        assert torch.equal(kept[..., :m].sort(-1).values.long(), best)
        assert torch.equal(kept[..., m:].long(), torch.arange(L - recent, L, device="cuda").expand(*kept.shape[:3], -1))
        rows = lambda p, n: p[:, :, was.long()].flatten(3, 4)[:, :, :, :n]     # [layers, 2, slots, n, heads, 64]
        at = kept.long().permute(0, 1, 3, 2)[:, None, :, :, :, None].expand(-1, 2, -1, -1, -1, 64)
        assert torch.equal(rows(pool, keep), rows(old, L).gather(3, at))
        assert torch.equal(w[..., :keep], w0.gather(-1, kept.long())) and not bool(w[..., keep:].any())
        del pool, old, kv
