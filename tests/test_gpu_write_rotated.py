"""New tokens that enter the cache (norm, rotation, write) against the same
steps in 64 bits.

Tolerance, per value: the result is rounded once (unit roundoff u), and before
that in 32 bits: the mean of D squares (D + 4 roundings of 2^-24, halved by the
root), root, quotient and two products, then the angle's reduction to [-pi, pi]
(2^-23 of it, and 2^-53 of the unreduced one), sine and cosine to 2^-22, and a
sum of two products.  With x1, x2 the normed values of the pair:
    |y - y64| <= u |y| + ((D / 2 + 12) 2^-24 + 2^-20 + 2^-52 |a|) (|x1| + |x2|).
Values that do not turn have no second one.  V is copied."""
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


class Case:
    def __init__(self, torch, n, heads, kv_heads, dim, pairs, page, dtype="bfloat16", norm=True, seed=0, layers=2,
                 far=0, std=1.0):
        from paper_2609_09800_amd import hbf
        self.torch, self.dtype, self.dim, self.pairs, self.page = torch, dtype, dim, pairs, page
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        dt = getattr(torch, dtype)
        lens = rng.integers(1, 60, 4) + -(-n // 4)
        held = -(-lens // page)
        pages = int(held.sum()) + 2
        perm = rng.permutation(pages).astype(np.int32)
        self.tables = np.full((5, int(held.max()) + 1), -1, np.int32)
        at = 0
        for s in range(4):
            self.tables[s, :held[s]] = perm[at:at + held[s]]
            at += held[s]
        places = np.array([(s, p) for s in range(4) for p in range(lens[s])], np.int32)
        places = places[rng.permutation(len(places))[:n]]
        self.slots, self.pos = places[:, 0].copy(), places[:, 1].copy()
        self.positions = self.pos + np.int32(far)
        self.freqs = 10000.0 ** (-np.arange(pairs) / max(pairs, 1))
        self.pool = torch.randn((layers, 2, pages, page, kv_heads, dim), generator=gen, device="cuda").to(dt)
        self.qkv = (torch.randn((n, heads + 2 * kv_heads, dim), generator=gen, device="cuda") * std).to(dt)
        self.q, self.k, self.v = self.qkv[:, :heads], self.qkv[:, heads:heads + kv_heads], self.qkv[:, heads + kv_heads:]
        self.w = [(1 + torch.randn(dim, generator=gen, device="cuda") * 0.3).to(dt) if norm else None for _ in range(2)]
        c = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.lens = lens.astype(np.int32)
        self.dev = dict(tables=c(self.tables), refs=c(np.ones(pages, np.int32)), lens=c(np.append(self.lens, np.int32(0))),
                        slots=c(self.slots), pos=c(self.pos), positions=c(self.positions), freqs=c(self.freqs))
        self.kv = hbf.KvPages(self.pool, refs=self.dev["refs"], tables=self.dev["tables"], lens=self.dev["lens"])

    def call(self, q_out, layer=1, **more):
        how = dict(q_weight=self.w[0], k_weight=self.w[1], eps=1e-5, positions=self.dev["positions"])
        how.update(more)
        return self.kv.write_rotated(layer, self.q, self.k, self.v, self.dev["slots"], self.dev["pos"], self.dev["freqs"],
                                     q_out, **how)

    def reference(self, x, weight, interleaved, eps=1e-5):
        """(y, |x1| + |x2| of the pair, the angles' size) in 64 bits."""
        torch = self.torch
        x = x.cpu().double()
        if weight is not None:
            x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.cpu().double()
        a = torch.from_numpy(self.positions.astype(np.float64)[:, None] * self.freqs)[:, None]
        y, size, angle = x.clone(), x.abs(), torch.zeros_like(x)
        p = self.pairs
        one, two = (slice(0, 2 * p, 2), slice(1, 2 * p, 2)) if interleaved else (slice(0, p), slice(p, 2 * p))
        y[..., one] = x[..., one] * a.cos() - x[..., two] * a.sin()
        y[..., two] = x[..., one] * a.sin() + x[..., two] * a.cos()
        for s in (one, two):
            size[..., s] = x[..., one].abs() + x[..., two].abs()
            angle[..., s] = a.abs().expand_as(angle[..., s])
        return y, size, angle

    def check(self, got, ref):
        y, size, angle = ref
        tol = U[self.dtype] * y.abs() + ((self.dim / 2 + 12) * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -52 * angle) * size
        if self.dtype == "float16":   # its smallest step
            tol = tol + 2.0 ** -25
        err = (got.cpu().double() - y).abs()
        assert bool((err <= tol).all()), f"worst {float((err / tol.clamp(min=1e-300)).max()):.3g} of the bound"


CASES = [
    # tokens, heads, kv heads, dim, pairs, page, far
    (1, 32, 4, 128, 64, 16, 0), (3, 1, 1, 64, 32, 1, 0), (77, 6, 2, 64, 16, 24, 1 << 20), (130, 8, 8, 128, 8, 16, 0),
    (5, 3, 1, 128, 0, 7, 0), (65, 40, 8, 64, 24, 64, -40), (33, 7, 7, 128, 56, 256, 1 << 30), (200, 64, 1, 128, 64, 16, 0),
    (300, 30, 3, 128, 40, 3, 5000),   # (enough for a wave per token)
]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_against_64_bits(torch, case, dtype, norm, interleaved):
    n, heads, kv_heads, dim, pairs, page, far = case
    say(f"write_rotated {case} {dtype} {norm} {interleaved}")
    c = Case(torch, n, heads, kv_heads, dim, pairs, page, dtype, norm, seed=n + dim, far=far)
    before = c.pool.clone()
    out = torch.full((n, heads, dim), 7.0, dtype=c.q.dtype, device="cuda")
    assert c.call(out, interleaved=interleaved) == OK
    assert c.kv.get_status() == OK
    c.check(out, c.reference(c.q, c.w[0], interleaved))
    page_of = torch.from_numpy(c.tables[c.slots, c.pos // page].astype(np.int64))
    at = torch.from_numpy((c.pos % page).astype(np.int64))
    c.check(c.pool[1, 0].cpu()[page_of, at], c.reference(c.k, c.w[1], interleaved))
    assert torch.equal(c.pool[1, 1].cpu()[page_of, at], c.v.cpu())
    # nothing else has changed
    want = before.cpu()
    want[1, :, page_of, at] = c.pool.cpu()[1, :, page_of, at]
    assert torch.equal(c.pool.cpu(), want)


def test_one_norm_of_two(torch):
    for one in (0, 1):
        c = Case(torch, 30, 4, 2, 64, 16, 16, seed=one)
        c.w[one] = None
        out = torch.empty((30, 4, 64), dtype=c.q.dtype, device="cuda")
        assert c.call(out) == OK
        c.check(out, c.reference(c.q, c.w[0], False))
        page_of = torch.from_numpy(c.tables[c.slots, c.pos // 16].astype(np.int64))
        c.check(c.pool[1, 0].cpu()[page_of, torch.from_numpy((c.pos % 16).astype(np.int64))], c.reference(c.k, c.w[1], False))


def test_in_place_and_wider_strides(torch):
    """Queries that turn where they lie; an output inside a wider tensor; positions that are the places."""
    for n in (1, 40, 300):
        say(f"write_rotated in place {n}")
        c = Case(torch, n, 12, 4, 128, 32, 16, seed=n)
        want = torch.empty((n, 12, 128), dtype=c.q.dtype, device="cuda")
        assert c.call(want) == OK
        pool = c.pool.clone()
        wide = torch.full((n, 2, 12, 136), 5.0, dtype=c.q.dtype, device="cuda")
        assert c.call(wide[:, 1, :, :128]) == OK
        assert torch.equal(wide[:, 1, :, :128], want) and bool((wide[:, 0] == 5.0).all()) and bool((wide[..., 128:] == 5.0).all())
        rest = c.qkv[:, 12:].clone()
        assert c.call(c.q, positions=None) == OK   # (here positions are the places)
        assert torch.equal(c.q, want) and torch.equal(c.qkv[:, 12:], rest) and torch.equal(c.pool, pool)
        assert c.kv.get_status() == OK


def test_zero_rows_and_values_that_are_not_finite(torch):
    """A head of zeros stays zero under a norm (eps 0: NaN, as 0 / 0 is); infinity and NaN stay in their head."""
    c = Case(torch, 20, 4, 2, 64, 32, 16, seed=3)
    want = torch.empty((20, 4, 64), dtype=c.q.dtype, device="cuda")
    assert c.call(want) == OK
    c.q[5, 1] = 0.0
    c.q[6, 2, 7] = float("nan")
    c.q[7, 3, 8] = float("inf")
    out = torch.empty_like(want)
    assert c.call(out) == OK
    ok = torch.ones((20, 4), dtype=torch.bool, device="cuda")
    ok[5, 1] = ok[6, 2] = ok[7, 3] = False
    assert torch.equal(out[ok], want[ok]) and bool((out[5, 1] == 0).all()) and bool(torch.isnan(out[6, 2]).all())
    assert bool(torch.isnan(out[7, 3]).any())
    assert c.call(out, eps=0.0) == OK and bool(torch.isnan(out[5, 1]).all())


def test_large_positions(torch):
    """Positions over all of 32 bits: the angle is taken in 64."""
    for far in (2 ** 31 - 400, -2 ** 31, -1):
        c = Case(torch, 50, 4, 2, 128, 64, 16, seed=4, far=far)
        out = torch.empty((50, 4, 128), dtype=c.q.dtype, device="cuda")
        assert c.call(out, interleaved=True) == OK
        c.check(out, c.reference(c.q, c.w[0], True))


@pytest.mark.parametrize("n", [1, 50, 400])
def test_bad_entries_are_left_out(torch, n):
    """Slots, places and pages out of range: no token of them enters the cache, the error stays until it is read."""
    say(f"write_rotated bad {n}")
    c = Case(torch, n, 4, 2, 64, 32, 16, seed=n + 5)
    want = torch.empty((n, 4, 64), dtype=c.q.dtype, device="cuda")
    clean = c.pool.clone()
    assert c.call(want) == OK
    full = c.pool.clone()
    at = n // 2
    s, p = int(c.slots[at]), int(c.pos[at])
    page, off = int(c.tables[s, p // 16]), p % 16
    for what in ("slot", "slot_low", "pos", "pos_low", "page", "page_low", "len"):
        c.pool.copy_(clean)
        saved = {k: c.dev[k].clone() for k in ("slots", "pos", "tables", "lens")}
        left_out = torch.zeros(n, dtype=torch.bool)
        left_out[at] = True
        if what.startswith("slot"):
            c.dev["slots"][at] = -1 if what == "slot_low" else len(c.tables)
        elif what.startswith("pos"):
            c.dev["pos"][at] = -1 if what == "pos_low" else int(c.lens[s])
        elif what.startswith("page"):
            c.dev["tables"][s, p // 16] = -1 if what == "page_low" else c.pool.shape[2]
            left_out = torch.from_numpy((c.slots == s) & (c.pos // 16 == p // 16))
        else:
            c.dev["lens"][s] = c.tables.shape[1] * 16 + 1
            left_out = torch.from_numpy(c.slots == s)
        out = torch.empty_like(want)
        assert c.call(out) == OK
        assert c.kv.get_status() == EINVAL and c.kv.get_status() == OK
        assert torch.equal(out, want)
        expect = full.clone()
        for j in torch.nonzero(left_out).flatten().tolist():
            pj, oj = int(c.tables[c.slots[j], c.pos[j] // 16]), int(c.pos[j]) % 16
            expect[1, :, pj, oj] = clean[1, :, pj, oj]
        assert torch.equal(c.pool, expect), what
        for k, v in saved.items():
            c.dev[k].copy_(v)


def test_refusals(torch):
    from paper_2609_09800_amd import hbf
    c = Case(torch, 9, 4, 2, 64, 16, 16, seed=6)
    d, out = c.dev, torch.empty((9, 4, 64), dtype=torch.bfloat16, device="cuda")
    a = (1, c.q, c.k, c.v, d["slots"], d["pos"], d["freqs"], out)

    def swap(i, x):
        return (*a[:i], x, *a[i + 1:])

    before = c.pool.clone()
    for args, how in ((swap(0, 2), {}), (swap(0, -1), {}), (swap(1, c.q.half()), {}), (swap(2, c.k[:, :1]), {}),
                      (swap(3, c.v[:8]), {}), (swap(4, d["slots"].long()), {}), (swap(5, d["pos"][:8]), {}),
                      (swap(6, d["freqs"].float()), {}), (swap(6, d["freqs"].cpu()), {}), (swap(7, out[:, :3]), {}),
                      (swap(7, out.float()), {}), (swap(1, c.q.cpu()), {}), (swap(7, out[:1].expand(9, -1, -1)), {}),
                      (swap(1, c.q[..., :32]), {}),
                      (a, dict(q_weight=c.w[0][:32])), (a, dict(k_weight=c.w[1].float())), (a, dict(positions=d["pos"].long()))):
        with pytest.raises(hbf.HbfError):
            c.kv.write_rotated(*args, **how)
    odd = torch.empty((9, 4, 68), dtype=torch.bfloat16, device="cuda")[..., :64]   # strides that are no multiples of 8
    for args, how in ((a, dict(eps=-1.0)), (a, dict(eps=float("nan"))), (swap(6, d["freqs"][:7]), {}),
                      (swap(6, torch.zeros(40, dtype=torch.float64, device="cuda")), {})):
        assert c.kv.write_rotated(*args, **how) == EINVAL
    try:
        assert c.kv.write_rotated(*swap(7, odd)) == EINVAL
    except hbf.HbfError:
        pass
    none = (1, c.q[:0], c.k[:0], c.v[:0], d["slots"][:0], d["pos"][:0], d["freqs"], out[:0])
    assert c.kv.write_rotated(*none) == OK and c.kv.get_status() == OK
    assert torch.equal(c.pool, before)


def test_offsets_past_32_bits(torch):
    """Places behind 2^32 bytes of a 9 GiB pool."""
    from paper_2609_09800_amd import hbf
    c = Case(torch, 40, 4, 4, 64, 32, 1024, seed=7)
    out = torch.empty((40, 4, 64), dtype=torch.bfloat16, device="cuda")
    assert c.call(out) == OK
    pages = 9000
    pool = torch.zeros((1, 2, pages, 1024, 4, 64), dtype=torch.bfloat16, device="cuda")
    moved = pages - c.pool.shape[2]
    tables = torch.where(c.dev["tables"] >= 0, c.dev["tables"] + moved, -1).int()
    kv = hbf.KvPages(pool, refs=torch.ones(pages, dtype=torch.int32, device="cuda"), tables=tables, lens=c.dev["lens"])
    c.kv, again = kv, torch.empty_like(out)
    assert c.call(again, layer=0) == OK and kv.get_status() == OK and torch.equal(out, again)
    page_of, at = tables.long()[c.slots, c.pos // 1024], torch.from_numpy((c.pos % 1024).astype(np.int64)).cuda()
    old = torch.from_numpy(c.tables[c.slots, c.pos // 1024].astype(np.int64)).cuda()
    assert torch.equal(pool[0][:, page_of, at], c.pool[1][:, old, at]) and not bool(pool[:, :, :moved].any())


def test_another_stream_and_graph(torch):
    for n in (1, 300):
        say(f"write_rotated graph {n}")
        c = Case(torch, n, 8, 2, 128, 64, 16, seed=8)
        want, out = (torch.empty((n, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        assert c.call(want) == OK
        pool = c.pool.clone()
        c.pool.zero_()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        assert c.call(out, stream=s) == OK
        s.synchronize()
        assert torch.equal(out, want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            assert c.call(out) == OK
        x = c.qkv.clone()
        for i in range(4):
            c.qkv.copy_(x * (i + 1))
            out.fill_(7.0)
            c.pool.zero_()
            g.replay()
            torch.cuda.synchronize()
            got = c.pool.clone()
            c.pool.zero_()
            assert c.call(want) == OK
            assert torch.equal(out, want) and torch.equal(got, c.pool)


def test_largest_calls(torch):
    """2^20 tokens, and 1,024 heads of each kind; without norms, turned by nothing: copies."""
    from paper_2609_09800_amd import hbf
    i32 = dict(dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(10)
    for n, heads, kv_heads, page in ((1 << 20, 2, 1, 16), (5, 1024, 1024, 4)):
        say(f"write_rotated largest {n} {heads}/{kv_heads}")
        held = -(-n // page)
        pool = torch.zeros((1, 2, held, page, kv_heads, 64), dtype=torch.float16, device="cuda")
        tables = torch.arange(held, **i32).flip(0).view(1, held).contiguous()
        kv = hbf.KvPages(pool, refs=torch.ones(held, **i32), tables=tables, lens=torch.full((1,), n, **i32))
        q, k, v = (torch.randn((n, h, 64), generator=gen, device="cuda").half() for h in (heads, kv_heads, kv_heads))
        out = torch.empty_like(q)
        freqs = torch.zeros(32, dtype=torch.float64, device="cuda")
        slots = torch.zeros(n, **i32)
        assert kv.write_rotated(0, q, k, v, slots, torch.arange(n, **i32), freqs, out) == OK and kv.get_status() == OK
        assert torch.equal(out, q)
        for plane, x in ((0, k), (1, v)):
            assert torch.equal(pool[0, plane][tables[0].long()].flatten(0, 1)[:n], x)
        del pool, q, k, v, out, kv
