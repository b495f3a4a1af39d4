"""Attention of new tokens over cache pages, and the weights it adds up, against
the same sums in 64 bits.

Tolerance, per element, from the formula o = sum p v, |v| weighted: the
result is rounded once and every p once to the 16-bit type (unit roundoff u),
and the scores carry the fp32 products' rounding, D * 2^-23 of sum |q k| scale,
which p turns into a relative error:
    |o - o64| <= u |o| + (u + 2 ds + (n + 16) 2^-23) sum p |v|,
    ds = (D + 8) 2^-23 max sum |q k| scale;  |lse - lse64| <= ds + (n + 16) 2^-23 + 2^-22 |lse|.
A token's weight is a sum of probabilities that are not rounded to 16 bits: each
is exp of a difference of two scores, divided by a sum, so it is off by
    p (4 ds + (n + 32) 2^-23) + 2^-23
(the last for the difference's own rounding, 2^-24 |x| e^-x <= 2^-24), and a
sum of Q of them and of what was there before adds (Q + 4) 2^-24 of itself.
"""
import math
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

OK, EINVAL = 0, -1
U = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


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


class Batch:
    """A cache of one layer, rows of new tokens, and what lies behind the lengths NaN and infinity."""

    def __init__(self, torch, heads, kv_heads, dim, new, lens, page, dtype="bfloat16", seed=0, q_std=2.0, slots=None,
                 extra=3, cols=0, tail=0, head=0):
        from paper_2609_09800_amd import hbf
        self.torch, self.dim, self.page, self.dtype = torch, dim, page, dtype
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        rng = np.random.default_rng(seed)
        dt = getattr(torch, dtype)
        n_slots = len(lens) + 1
        self.slots = rng.permutation(n_slots)[:len(lens)].astype(np.int32) if slots is None else np.array(slots, np.int32)
        self.lens = np.array(lens, np.int32)
        by_slot = np.zeros(n_slots, np.int32)
        for s, n in zip(self.slots, lens):
            by_slot[s] = n
        held = -(-by_slot // page)
        pages = int(held.sum()) + extra
        perm = rng.permutation(pages).astype(np.int32)
        self.tables = np.full((n_slots, int(held.max()) + 1 + cols), -1, np.int32)
        at = 0
        for s in range(n_slots):
            self.tables[s, :held[s]] = perm[at:at + held[s]]
            at += held[s]
        pool = torch.randn((1, 2, pages, page, kv_heads, dim), generator=gen, device="cuda").to(dt)
        bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda").to(dt)
        fill = bad[torch.arange(kv_heads * dim, device="cuda") % 3].view(kv_heads, dim)
        pool[:, :, torch.from_numpy(perm[at:]).cuda().long()] = fill
        for s in range(n_slots):
            if by_slot[s] % page:
                pool[:, :, int(self.tables[s, held[s] - 1]), int(by_slot[s]) % page:] = fill
        self.pool = pool
        self.new = np.array(new, np.int32)
        self.starts = (head + np.concatenate([[0], np.cumsum(self.new)])).astype(np.int32)
        tokens = int(self.starts[-1]) + tail
        self.q = (torch.randn((tokens, heads, dim), generator=gen, device="cuda") * q_std).to(dt)
        self.weights = torch.rand((n_slots, kv_heads, self.tables.shape[1] * page), generator=gen, device="cuda")
        c = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.dev = dict(tables=c(self.tables), refs=c(np.ones(pages, np.int32)), lens=c(by_slot), slots=c(self.slots),
                        starts=c(self.starts))
        self.kv = hbf.KvPages(pool, refs=self.dev["refs"], tables=self.dev["tables"], lens=self.dev["lens"])

    def run(self, weights=None, **how):
        torch = self.torch
        out = torch.full_like(self.q, 7.0)
        lse = torch.full(self.q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
        rc = self.kv.attention(0, self.q, out, self.dev["slots"], self.dev["starts"], lse=lse, weights=weights, **how)
        assert rc == OK
        return out, lse

    def reference(self, scale=None, window=0, sinks=0, weights=None):
        """(out, lse, sum p|v|, ds, weights, their bounds) in 64 bits on the CPU; 7 where no row is."""
        torch = self.torch
        q, pool = self.q.cpu().double(), self.pool[0].cpu().double()
        T, Hq, D = q.shape
        Hk = pool.shape[3]
        scale = D ** -0.5 if scale is None else scale
        out, mag = torch.full((T, Hq, D), 7.0, dtype=torch.float64), torch.zeros((T, Hq, D), dtype=torch.float64)
        lse, ds = torch.full((T, Hq), 7.0, dtype=torch.float64), torch.zeros((T, Hq), dtype=torch.float64)
        wsum = None if weights is None else weights.cpu().double()
        wtol = None if weights is None else torch.zeros_like(wsum)
        count = None if weights is None else torch.zeros_like(wsum)
        for i, slot in enumerate(self.slots):
            L = int(self.dev["lens"][int(slot)])
            s0, n = int(self.starts[i]), int(self.new[i])
            kv = pool[:, torch.from_numpy(self.tables[slot, :-(-L // self.page)]).long()].reshape(2, -1, Hk, D)[:, :L]
            pos = torch.arange(L - n, L)
            j = torch.arange(L)
            seen = j[None, :] <= pos[:, None]
            if window:
                seen &= (j[None, :] > pos[:, None] - window) | (j[None, :] < sinks)
            for h in range(Hq):
                if n == 0:
                    continue
                g = h // (Hq // Hk)
                k, v = kv[0, :, g], kv[1, :, g]
                s = (q[s0:s0 + n, h] @ k.t()) * scale
                s = s.masked_fill(~seen, -math.inf)
                m = s.max(-1, keepdim=True)[0] if L else torch.full((n, 1), -math.inf, dtype=torch.float64)
                e = torch.where(seen, torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
                l = e.sum(-1, keepdim=True)
                p = e / torch.where(l == 0, 1.0, l)
                big = ((q[s0:s0 + n, h].abs() @ k.abs().t()) * abs(scale) * seen).amax(-1) if L else torch.zeros(n).double()
                rows = slice(s0, s0 + n)
                ds[rows, h] = (D + 8) * 2.0 ** -23 * big
                lse[rows, h] = torch.where(l == 0, -math.inf, torch.where(m == -math.inf, 0.0, m) + l.log())[:, 0]
                # what a query does not see stays out, whatever it is
                for t in range(n) if not torch.isfinite(v).all() else [slice(None)]:
                    if isinstance(t, int):
                        keep = seen[t]
                        out[s0 + t, h] = p[t, keep] @ v[keep]
                        mag[s0 + t, h] = p[t, keep] @ v[keep].abs()
                    else:
                        out[rows, h], mag[rows, h] = p @ v, p @ v.abs()
                if weights is not None:
                    wsum[slot, g, :L] += p.sum(0)
                    wtol[slot, g, :L] += (p * (4 * ds[rows, h, None] + (L + 32) * 2.0 ** -23) + seen * 2.0 ** -23).sum(0)
                    count[slot, g, :L] += seen.sum(0)
        if weights is not None:
            wtol += torch.where(count > 0, (count + 4) * 2.0 ** -24 * wsum, 0.0)
        return out, lse, mag, ds, wsum, wtol

    def check(self, got, got_lse, ref, got_weights=None):
        torch = self.torch
        out, lse, mag, ds, wsum, wtol = ref
        u, n = U[self.dtype], int(self.lens.max(initial=0))
        tol = u * out.abs() + (u + 2 * ds[..., None] + (n + 16) * 2.0 ** -23) * mag
        g = got.cpu().double()
        fin = torch.isfinite(out)
        assert bool((torch.isfinite(g) == fin).all()), "finite where the sums are"
        err = (g - out).abs()
        assert bool((err <= tol)[fin].all()), f"out: worst {float((err / tol.clamp(min=1e-300))[fin].max()):.3g} of the bound"
        g = got_lse.cpu().double()
        none = lse == -math.inf
        assert bool(((g == -math.inf) == none).all())
        tl = ds + (n + 16) * 2.0 ** -23 + 2.0 ** -22 * lse.abs()
        assert bool(((g - lse).abs() <= tl)[~none].all()), "lse"
        if got_weights is not None:
            err = (got_weights.cpu().double() - wsum).abs()
            assert bool((err <= wtol).all()), f"weights: worst {float((err / wtol.clamp(min=1e-300)).max()):.3g} of the bound"


CASES = [
    # heads, kv heads, dim, new tokens, lengths, page, window, sinks
    (8, 1, 128, [1], [1], 16, 0, 0),
    (1, 1, 64, [1], [33], 8, 0, 0),
    (4, 4, 64, [1, 1], [0, 5], 16, 0, 0),                          # a query at position -1
    (6, 2, 128, [1, 1, 1], [1, 700, 64], 24, 0, 0),
    (16, 1, 64, [2, 0, 3, 1], [129, 17, 3, 1], 1, 0, 0),
    (64, 2, 128, [1, 2], [1000, 40], 7, 0, 0),
    (6, 2, 64, [130, 0, 3, 24, 25], [130, 9, 99, 24, 500], 24, 0, 0),
    (8, 2, 128, [70], [70], 16, 0, 0),                              # a prompt from its start
    (8, 1, 128, [50, 1, 1], [600, 2000, 3], 16, 0, 0),              # a chunk and single tokens in one call
    (32, 4, 128, [33], [2000], 16, 0, 0),
    (4, 4, 64, [200], [333], 64, 0, 0),
    (3, 1, 128, [9, 5], [4, 5], 256, 0, 0),                         # fewer tokens in the cache than new ones
    (48, 1, 128, [1, 7], [640, 1000], 16, 0, 0),
    (20, 1, 64, [1, 1], [513, 64], 32, 0, 0),
    (32, 4, 128, [1], [20000], 16, 0, 0),
    (8, 2, 128, [1, 1, 1], [1000, 3, 70], 16, 64, 4),               # windows
    (8, 2, 128, [100, 30], [1000, 45], 16, 64, 4),
    (4, 1, 64, [150], [150], 16, 1, 0),
    (4, 1, 64, [150], [700], 16, 1, 1),
    (8, 1, 128, [40], [900], 16, 17, 200),                          # more first tokens than the window
    (16, 2, 64, [300], [301], 24, 128, 33),
    (8, 2, 128, [64], [2000], 16, 5000, 4),                         # a window past the length
    (8, 2, 64, [10], [400], 16, 2 ** 31 - 1, 2 ** 31 - 1),
]



# In tables that could hold 19,200 tokens more: such calls are cut into tiles of 256 queries.
WIDE_CASES = [
    (12, 4, 64, [130, 0, 3, 24, 25], [130, 9, 99, 24, 500], 24, 0, 0),
    (32, 8, 128, [70], [70], 16, 0, 0),
    (64, 8, 128, [50, 1, 1], [600, 2000, 3], 16, 0, 0),
    (64, 8, 128, [33], [2000], 1, 0, 0),
    (8, 8, 64, [200], [333], 64, 0, 0),
    (24, 8, 128, [19, 5], [4, 5], 256, 0, 0),       # more new tokens than there are
    (32, 8, 128, [100, 30], [1000, 45], 16, 64, 4),
    (8, 8, 64, [150], [150], 16, 1, 0),
    (8, 8, 64, [150], [700], 16, 1, 1),
    (64, 8, 128, [40], [900], 7, 17, 200),
    (64, 8, 64, [300], [301], 24, 128, 33),
    (32, 8, 128, [64], [2000], 16, 5000, 4),
    (32, 8, 64, [30], [400], 16, 2 ** 31 - 1, 2 ** 31 - 1),
    (64, 8, 128, [64], [5000], 16, 0, 0),           # in parts
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case,cols", [(c, 0) for c in CASES] + [(c, 19200) for c in WIDE_CASES],
                         ids=lambda c: "-".join(map(str, c)).replace(" ", "") if isinstance(c, tuple) else str(c))
def test_against_64_bits(torch, case, cols, dtype):
    heads, kv_heads, dim, new, lens, page, window, sinks = case
    say(f"attention {case} {dtype} {cols}")
    b = Batch(torch, heads, kv_heads, dim, new, lens, page, dtype, seed=sum(lens), tail=2, head=1, cols=cols // page)
    for weights in (None, b.weights):
        got_w = None if weights is None else weights.clone()
        out, lse = b.run(weights=got_w, window=window, sinks=sinks)
        assert b.kv.get_status() == OK
        b.check(out, lse, b.reference(window=window, sinks=sinks, weights=weights), got_w)
    scores = b.q.shape[0] * heads * b.weights.shape[-1] * 4   # bytes that tiles of 16 would leave
    assert not cols or scores > 512 << 20 or b.kv._chunk_bytes < scores, "tiles of 256"


# heads, kv heads, dim, new tokens, lengths, page, extra columns: tiles of 16, one a row or more; of 256, in parts
SHAPES = [(8, 2, 64, [1, 1, 2], [40, 300, 7], 16, 0), (8, 2, 128, [30, 1], [200, 77], 16, 0),
          (16, 4, 128, [60, 20], [2100, 30], 16, 1200), (8, 8, 64, [300], [1200], 24, 800)]
IDS = [f"{s[0]}x{s[2]}-{s[6]}" for s in SHAPES]


def batch(torch, shape, **how):
    heads, kv_heads, dim, new, lens, page, cols = shape
    return Batch(torch, heads, kv_heads, dim, new, lens, page, cols=cols, **how)


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("scale,q_std", [(0.0, 1.0), (-0.3, 1.0), (0.5, 8.0), (1e-3, 0.1)])
def test_scales(torch, scale, q_std, shape):
    """Flat, reversed and nearly one-hot softmaxes."""
    say(f"attention scale {scale} {shape}")
    b = batch(torch, shape, seed=3, q_std=q_std)
    w = b.weights.clone()
    out, lse = b.run(scale=scale, weights=w)
    b.check(out, lse, b.reference(scale=scale, weights=b.weights), w)


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("up", [1.0, -1.0])
def test_rising_scores(torch, up, shape):
    """The running maximum moves at every step, by far more than the type's range of exp."""
    say(f"attention rising {up} {shape}")
    b = batch(torch, shape, seed=4)
    for s, L in zip(b.slots, b.lens):
        for j in range(L):
            b.pool[0, 0, int(b.tables[s, j // b.page]), j % b.page, :, 0] = up * (60.0 * j / max(L, 1) - 30)
    b.q[:, :, 0] = 40.0
    w = b.weights.clone()
    out, lse = b.run(scale=0.125, weights=w)
    b.check(out, lse, b.reference(scale=0.125, weights=b.weights), w)


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("dtype,q_value,unit", [
    ("bfloat16", 2.0 ** 10, 2.0 ** 12), ("bfloat16", 2.0 ** 20, 2.0 ** 20), ("bfloat16", 2.0 ** 50, 2.0 ** 60),
    ("float16", 2.0 ** 10, 2.0 ** 8), ("float16", 2.0 ** 15, 2.0 ** 12)])
def test_scores_of_any_size(torch, dtype, q_value, unit, shape):
    """Scores of up to 2^118, far past where one step of a float is more than the range of exp: the highest
    tokens, and as many as tie, share the query.  (The scores are exact in 32 bits, so that ds is 0.)"""
    say(f"attention scores {dtype} {q_value} {unit} {shape}")
    b = batch(torch, shape, seed=31, dtype=dtype)
    keys = torch.randint(-7, 8, b.pool.shape[2:5], generator=torch.Generator(device="cuda").manual_seed(32), device="cuda")
    keep = torch.isfinite(b.pool[0, 0])   # (what lies behind the lengths stays NaN and infinity)
    b.pool[0, 0] = torch.where(keep, (keys[..., None] * unit).to(b.pool.dtype), b.pool[0, 0])
    b.q[:] = q_value
    w = b.weights.clone()
    out, lse = b.run(scale=0.125, weights=w)
    assert b.kv.get_status() == OK
    ref = list(b.reference(scale=0.125, weights=b.weights))
    n = max(b.lens) + 32
    ref[3] = torch.zeros_like(ref[3])
    ref[5] = b.reference(scale=0.0, weights=b.weights)[5] + n * 2.0 ** -23 * ref[4]   # (every p at most 1)
    b.check(out, lse, ref, w)


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 2)])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_what_a_query_does_not_see_stays_out(torch, value, window, sinks, shape):
    """K and V of some tokens are not finite: queries before them, and those whose window has passed them, are as ever."""
    say(f"attention not finite {value} {window} {shape}")
    b = batch(torch, shape, seed=5)
    clean = b.run(window=window, sinks=sinks)
    w0 = b.weights.clone()
    b.run(window=window, sinks=sinks, weights=w0)
    bad = {}
    for i, (s, L, n) in enumerate(zip(b.slots, b.lens, b.new)):
        bad[i] = [L - n // 2 - 1] if n > 1 else ([int(L) // 2] if window and L > 40 else [])
        for j in bad[i]:
            for plane in (0, 1):
                b.pool[0, plane, int(b.tables[s, j // b.page]), j % b.page, :, 3] = value
    w = b.weights.clone()
    out, lse = b.run(window=window, sinks=sinks, weights=w)
    assert b.kv.get_status() == OK
    for i, (s0, L, n, slot) in enumerate(zip(b.starts, b.lens, b.new, b.slots)):
        for t in range(n):
            p = L - n + t
            sees = any(j <= p and (not window or j > p - window or j < sinks) for j in bad[i])
            if not sees:   # (a tile that holds such a value takes its products in another order)
                for got, want in ((out, clean[0]), (lse, clean[1])):
                    g, c = got[s0 + t].double(), want[s0 + t].double()
                    assert bool(((g - c).abs() <= 2.0 ** -7 * (c.abs() + 1)).all())
        # tokens that only such queries see have their weights as ever
        if bad[i] and not window:
            first = L - n
            assert bool((w[slot, :, L:] == w0[slot, :, L:]).all())
            late = bad[i][0] + 1
            assert not bool(torch.isnan(out[s0:s0 + max(0, bad[i][0] - first)]).any())


def test_infinite_values_that_are_seen(torch):
    """V with infinity and NaN: the dimension that has it, of the queries that see it, and no other."""
    for shape in SHAPES:
        say(f"attention infinite values {shape}")
        b = batch(torch, shape, seed=6)
        s, L, n = int(b.slots[0]), int(b.lens[0]), int(b.new[0])
        j = L - max(n // 2, 1)
        b.pool[0, 1, int(b.tables[s, j // b.page]), j % b.page, :, 5] = math.inf
        out, lse = b.run()
        ref = b.reference()
        b.check(out, lse, ref)
        seen = out[int(b.starts[0]) + n - 1]
        assert bool(torch.isinf(seen[:, 5]).all()) and bool(torch.isfinite(seen[:, :5]).all())


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_nan_in_a_query_stays_there(torch, shape):
    b = batch(torch, shape, seed=7)
    want, want_lse = b.run()
    at = int(b.starts[1]) - 1 if len(b.new) > 1 else 3
    b.q[at, 1, 2] = math.nan
    out, lse = b.run()
    ok = torch.ones(out.shape[:2], dtype=torch.bool, device="cuda")
    ok[at, 1] = False
    assert bool(torch.isnan(out[at, 1]).all()) and torch.equal(out[ok], want[ok]) and torch.equal(lse[ok], want_lse[ok])


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_strides_and_layouts(torch, shape):
    """Queries and outputs inside wider tensors, weights of a layer inside all layers', tables and another layer of the pool."""
    from paper_2609_09800_amd import hbf
    say(f"attention layouts {shape}")
    b = batch(torch, shape, seed=8)
    w = b.weights.clone()
    want, want_lse = b.run(weights=w)
    T, H, D = b.q.shape
    two = torch.zeros((2, *b.pool.shape[1:]), dtype=b.pool.dtype, device="cuda")
    two[1] = b.pool[0]
    tables = torch.full((b.tables.shape[0], b.tables.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
    tables[:, :-3] = b.dev["tables"]
    kv = hbf.KvPages(two, refs=b.dev["refs"], tables=tables[:, :-3], lens=b.dev["lens"])
    wide = torch.full((T, 3, H, D + 8), 5.0, dtype=b.q.dtype, device="cuda")
    wide[:, 1, :, :D] = b.q
    out = torch.full((T, H, 2, D), 5.0, dtype=b.q.dtype, device="cuda")
    all_w = torch.full((b.weights.shape[0], 3, b.weights.shape[1], b.weights.shape[2] + 5), 5.0, device="cuda")
    all_w[:, 1, :, :-5] = b.weights
    lse = torch.empty_like(want_lse)
    assert kv.attention(1, wide[:, 1, :, :D], out[:, :, 1], b.dev["slots"], b.dev["starts"], lse=lse, weights=all_w[:, 1]) == OK
    assert torch.equal(out[:, :, 1], want) and torch.equal(lse, want_lse) and torch.equal(all_w[:, 1, :, :-5], w)
    assert bool((out[:, :, 0] == 5.0).all()) and bool((all_w[:, ::2] == 5.0).all()) and bool((all_w[..., -5:] == 5.0).all())
    # without lse; nothing to do
    o2 = torch.empty_like(b.q)
    assert kv.attention(1, b.q, o2, b.dev["slots"], b.dev["starts"]) == OK and torch.equal(o2, want)
    assert kv.attention(1, b.q, o2, b.dev["slots"][:0], b.dev["starts"][:1]) == OK and torch.equal(o2, want)
    assert kv.attention(1, b.q[:0], o2[:0], b.dev["slots"], torch.zeros_like(b.dev["starts"])) == OK
    assert kv.attention(1, b.q[:0], o2[:0], b.dev["slots"][:0], b.dev["starts"][:1], weights=all_w[:, 1]) == OK
    assert kv.attention(1, b.q[:1], o2[:1], b.dev["slots"][:0], b.dev["starts"][:1]) == OK
    assert kv.get_status() == OK


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_repeats_bit_for_bit_from_any_scratch(torch, shape):
    b = batch(torch, shape, seed=9)
    runs = []
    for fill in (0, 255, 255):
        if b.kv._attn_ws._t is not None:
            b.kv._attn_ws._t.fill_(fill)
        w = b.weights.clone()
        runs.append((*b.run(weights=w), w))
        assert not bool(b.kv._chunk_ctl.any())
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))
    # without control words nothing is cut into parts
    b.kv._chunk_at = None
    w = b.weights.clone()
    out, lse = b.run(weights=w)
    b.check(out, lse, b.reference(weights=b.weights), w)


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_rows_of_one_slot(torch, shape):
    """A slot that several rows name: each result as alone, its weights the sum of all."""
    heads, kv_heads, dim, new, lens, page, cols = shape
    say(f"attention rows of one slot {shape}")
    L = max(lens)
    b = Batch(torch, heads, kv_heads, dim, [new[0], 3, new[0]], [L, 50, L], page, cols=cols, seed=10, slots=[2, 0, 2])
    w = b.weights.clone()
    out, lse = b.run(weights=w)
    b.check(out, lse, b.reference(weights=b.weights), w)


def test_many_rows(torch):
    """More rows than are searched at a time, and than a workgroup has threads; rows without tokens among them."""
    rng = np.random.default_rng(11)
    for rows, top, cols in ((70, 3, 0), (4200, 2, 0), (600, 40, 3000), (300, 60, 3000)):
        say(f"attention {rows} rows")
        new = rng.integers(0, top, rows)
        lens = np.maximum(new, rng.integers(0, 9, rows))
        b = Batch(torch, 2, 1, 64, new, lens, 8, seed=rows, cols=cols)
        w = b.weights[:, :, :64].contiguous()   # (no token lies behind)
        got = w.clone()
        out, lse = b.run(weights=got)
        assert b.kv.get_status() == OK
        b.check(out, lse, b.reference(weights=w), got)


@pytest.mark.parametrize("heads,kv_heads,dim,new", [(8, 2, 64, [1, 1, 2]), (8, 2, 128, [14, 1])])
def test_weights_beside_tables_of_millions_of_tokens(torch, heads, kv_heads, dim, new):
    """Scores of all that the tables could hold would take more scratch than is given to them."""
    say(f"attention wide tables {heads} {dim}")
    for cols, dtype in ((20, "float16"), (9000, "bfloat16")):
        b = Batch(torch, heads, kv_heads, dim, new, [70, 900, 30][:len(new)], 1024, dtype=dtype, seed=17, cols=cols)
        w = b.weights.clone()
        out, lse = b.run(weights=w, window=200, sinks=5)
        b.check(out, lse, b.reference(window=200, sinks=5, weights=b.weights), w)
        need = b.q.shape[0] * heads * b.weights.shape[-1] * 4
        assert (need > 512 << 20) == (b.kv._chunk_bytes < need), "the scratch is what the scores say"


def test_offsets_past_32_bits(torch):
    """Pages behind 2^32 bytes of a 9 GiB pool."""
    from paper_2609_09800_amd import hbf
    for new, lens in (([1, 1], [100, 1500]), ([40, 9], [300, 1100])):
        b = Batch(torch, 8, 4, 64, new, lens, 1024, seed=12, cols=100)
        want = b.run()
        pages = 9000
        pool = torch.zeros((1, 2, pages, 1024, 4, 64), dtype=torch.bfloat16, device="cuda")
        moved = pages - b.pool.shape[2]
        pool[:, :, moved:] = b.pool
        tables = torch.where(b.dev["tables"] >= 0, b.dev["tables"] + moved, -1).int()
        kv = hbf.KvPages(pool, refs=torch.ones(pages, dtype=torch.int32, device="cuda"), tables=tables, lens=b.dev["lens"])
        out = torch.empty_like(b.q)
        w, w2 = b.weights.clone(), b.weights.clone()
        assert kv.attention(0, b.q, out, b.dev["slots"], b.dev["starts"], weights=w) == OK
        b.run(weights=w2)
        assert torch.equal(out, want[0]) and torch.equal(w, w2)
        del pool, kv


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("what", ["long", "negative", "weights", "slot", "slot_low", "page", "page_low"])
def test_bad_entries_fail_closed(torch, what, shape):
    """A slot, length or page out of range: that row is NaN, the others are right."""
    say(f"attention bad {what} {shape}")
    heads, kv_heads, dim, new, lens, page, cols = shape
    b = Batch(torch, heads, kv_heads, dim, [new[0], new[0], 2], [lens[0], lens[0] + 30, 20], page, cols=cols, seed=13)
    want, want_lse = b.run()
    s = int(b.slots[1])
    weights = b.weights.clone()
    if what == "long":
        b.dev["lens"][s] = b.tables.shape[1] * page + 1
    elif what == "negative":
        b.dev["lens"][s] = -1
    elif what == "weights":
        weights = weights[:, :, :lens[0] + 29].contiguous()
    elif what == "slot":
        b.dev["slots"][1] = b.tables.shape[0]
    elif what == "slot_low":
        b.dev["slots"][1] = -1
    elif what == "page":
        b.dev["tables"][s, 0] = b.pool.shape[2]
    else:
        b.dev["tables"][s, 0] = -1
    w = weights.clone()
    out, lse = b.run(weights=w)
    assert b.kv.get_status() == EINVAL and b.kv.get_status() == OK
    rows = slice(int(b.starts[1]), int(b.starts[2]))
    keep = torch.ones(len(out), dtype=torch.bool, device="cuda")
    keep[rows] = False
    assert bool(torch.isnan(out[rows]).all()) and bool(torch.isnan(lse[rows]).all())
    assert torch.equal(out[keep], want[keep]) and torch.equal(lse[keep], want_lse[keep])
    assert torch.equal(w[s], weights[s])


def test_bad_starts(torch):
    """Starts that decrease or leave the queries: an error, and nothing outside the tensors is touched."""
    for shape in SHAPES:
        b = batch(torch, shape, seed=14)
        for change in ((1, -5), (1, 10 ** 9), (len(b.new), len(b.q) + 1), (0, int(b.starts[1]) + 1)):
            say(f"attention bad starts {change} {shape}")
            b.dev["starts"].copy_(torch.from_numpy(b.starts))
            b.dev["starts"][change[0]] = change[1]
            b.run(weights=b.weights.clone())
            assert b.kv.get_status() == EINVAL
            assert not bool(b.kv._chunk_ctl.any())


def test_refusals(torch):
    from paper_2609_09800_amd import hbf
    b = batch(torch, SHAPES[0], seed=15)
    out, lse = b.run()
    sl, st, q, w = b.dev["slots"], b.dev["starts"], b.q, b.weights
    for args, how in (((1, q, out, sl, st), {}), ((0, q.float(), out, sl, st), {}), ((0, q, out[:3], sl, st), {}),
                      ((0, q, out, sl, st[:-1]), {}), ((0, q, out, sl.long(), st), {}), ((0, q, out, sl, st.long()), {}),
                      ((0, q.cpu(), out, sl, st), {}), ((0, q, out[:1].expand(len(q), -1, -1), sl, st), {}),
                      ((0, q[..., :32], out[..., :32], sl, st), {}), ((0, q, out, sl, st), dict(lse=lse[:, :3])),
                      ((0, q, out, sl, st), dict(weights=w[:-1])), ((0, q, out, sl, st), dict(weights=w.double())),
                      ((0, q, out, sl, st), dict(weights=w[:, :1])), ((0, q, out, sl, st), dict(weights=w[:1].expand(len(w), -1, -1))),
                      ((0, q, out, sl, st), dict(weights=w[..., ::2]))):
        with pytest.raises(hbf.HbfError):
            b.kv.attention(*args, **how)
    with pytest.raises(hbf.HbfError):
        hbf.KvPages(b.pool).attention(0, q, out, sl, st)
    assert b.kv.attention(0, q[:, :7], out[:, :7], sl, st) == EINVAL     # 7 heads over 2
    for how in (dict(window=-1), dict(sinks=-1), dict(scale=math.nan), dict(scale=math.inf)):
        assert b.kv.attention(0, q, out, sl, st, **how) == EINVAL


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_another_stream_and_graph(torch, shape):
    say(f"attention graph {shape}")
    b = batch(torch, shape, seed=16)
    want, want_lse = b.run()
    out = torch.empty_like(b.q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    assert b.kv.attention(0, b.q, out, b.dev["slots"], b.dev["starts"], stream=s) == OK
    s.synchronize()
    assert torch.equal(out, want)
    q, out, lse = b.q.clone(), torch.empty_like(b.q), torch.empty_like(want_lse)
    w = torch.zeros_like(b.weights)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert b.kv.attention(0, b.q, out, b.dev["slots"], b.dev["starts"], lse=lse, weights=w) == OK
    lens = b.dev["lens"].clone()
    for i in range(4):   # other queries and lengths than were captured
        b.q.copy_(q * (i + 1) / 2)
        b.dev["lens"].copy_((lens - i).clamp(min=0))
        out.fill_(7.0)
        lse.fill_(7.0)
        w.fill_(0.5)
        g.replay()
        torch.cuda.synchronize()
        w2 = torch.full_like(w, 0.5)
        eager, eager_lse = b.run(weights=w2)
        rows = slice(int(b.starts[0]), int(b.starts[-1]))
        assert torch.equal(out[rows], eager[rows]) and torch.equal(lse[rows], eager_lse[rows]) and torch.equal(w, w2)


def test_largest_calls(torch):
    """As many rows, tokens, heads of a group and tokens of a page as a call takes.  Where a query sees its own
    token alone the result is that token's V, whose weight grows by one a query head."""
    from paper_2609_09800_amd import hbf
    gen = torch.Generator(device="cuda").manual_seed(18)
    i32 = dict(dtype=torch.int32, device="cuda")
    # rows, new tokens of each, heads, kv heads, page, window
    for rows, new, heads, kv_heads, page, window in ((65535, 1, 2, 1, 1, 0), (1, 1 << 20, 16, 2, 16, 1), (3, 5, 1024, 1, 65536, 1),
                                                     (2, 1, 1024, 1024, 4, 0), (512, 2048, 1, 1, 256, 1), (5000, 200, 1, 1, 8, 1)):
        say(f"attention largest {rows} {new} {heads}/{kv_heads} {page}")
        held = -(-new // page)
        pool = torch.randn((1, 2, rows * held, page, kv_heads, 64), generator=gen, device="cuda").bfloat16()
        tables = torch.arange(rows * held, **i32).view(rows, held).flip(0).contiguous()
        kv = hbf.KvPages(pool, refs=torch.ones(rows * held, **i32), tables=tables, lens=torch.full((rows,), new, **i32))
        q = torch.randn((rows * new, heads, 64), generator=gen, device="cuda").bfloat16()
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        w = torch.zeros((rows, kv_heads, new), device="cuda")
        slots, starts = torch.arange(rows, **i32), torch.arange(0, rows * new + 1, new, **i32)
        assert kv.attention(0, q, out, slots, starts, lse=lse, weights=w, window=window) == OK
        assert kv.get_status() == OK
        v = pool[0, 1][tables.long()].flatten(1, 2)[:, :new].flatten(0, 1)   # [rows * new, kv heads, 64]
        want = v.repeat_interleave(heads // kv_heads, 1)
        # the bounds above for one token: sum p |v| is |v|, and |q k| at most the product of both norms
        k = pool[0, 0][tables.long()].flatten(1, 2)[:, :new].flatten(0, 1)
        ds = (64 + 8) * 2.0 ** -23 * float(q.float().norm(dim=-1).max() * k.float().norm(dim=-1).max()) / 8
        bound = 2 * U["bfloat16"] + 2 * ds + 17 * 2.0 ** -23
        assert bool(((out.float() - want.float()).abs() <= bound * want.float().abs()).all())
        n = heads // kv_heads
        assert bool(((w - n).abs() <= n * (4 * ds + 34 * 2.0 ** -23) + (n + 4) * 2.0 ** -24 * n).all())
        del pool, q, out, want, v, k, kv
