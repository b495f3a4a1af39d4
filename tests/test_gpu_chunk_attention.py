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


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_against_64_bits(torch, case, dtype):
    heads, kv_heads, dim, new, lens, page, window, sinks = case
    say(f"attention {case} {dtype}")
    b = Batch(torch, heads, kv_heads, dim, new, lens, page, dtype, seed=sum(lens), tail=2, head=1)
    for weights in (None, b.weights):
        got_w = None if weights is None else weights.clone()
        out, lse = b.run(weights=got_w, window=window, sinks=sinks)
        assert b.kv.get_status() == OK
        b.check(out, lse, b.reference(window=window, sinks=sinks, weights=weights), got_w)
