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
            assert np.array_equal(self.dev[name].cpu().numpy(), getattr(self, name)), name
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
