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
