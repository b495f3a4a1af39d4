"""Attention over a shared prefix and own cache pages against the same sums in
64 bits.

Tolerance, per element, from the formula o = sum p v, |v| weighted: the
result is rounded once and every p once to the 16-bit type (unit roundoff u),
and the scores carry the fp32 products' rounding, D * 2^-23 of sum |q k| scale,
which p turns into a relative error:
    |o - o64| <= u |o| + (u + 2 ds + (n + 16) 2^-23) sum p |v|,
    ds = (D + 8) 2^-23 max sum |q k| scale;  |lse - lse64| <= ds + (n + 16) 2^-23 + 2^-22 |lse|.
"""
import math
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

OK, EINVAL, ENOWORKSPACE = 0, -1, -4


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


def reference(torch, pool, q, prefix, prefix_len, tables, lens, scale):
    """(out, lse, sum p|v|, max sum |q k| scale) in 64 bits on the CPU."""
    pool, q = pool.cpu().double(), q.cpu().double()
    pt, Hk, D = pool.shape[2:]
    R, Hq, _ = q.shape
    out, mag = torch.zeros((R, Hq, D), dtype=torch.float64), torch.zeros((R, Hq, D), dtype=torch.float64)
    lse, big = torch.full((R, Hq), -math.inf, dtype=torch.float64), torch.zeros((R, Hq), dtype=torch.float64)
    pre = pool[:, prefix.cpu().long()].reshape(2, -1, Hk, D)[:, :prefix_len] if prefix_len else pool[:, :0].reshape(2, 0, Hk, D)
    for r in range(R):
        n = int(lens[r]) if lens is not None else 0
        own = pool[:, tables[r, :-(-n // pt)].cpu().long()].reshape(2, -1, Hk, D)[:, :n] if n else pre[:, :0]
        k, v = torch.cat([pre, own], 1)
        if k.shape[0] == 0:
            continue
        for j in range(Hq):
            h = j // (Hq // Hk)
            s = (k[:, h] @ q[r, j]) * scale
            big[r, j] = (k[:, h].abs() @ q[r, j].abs()).max() * abs(scale)
            p = torch.softmax(s, 0)
            out[r, j], mag[r, j], lse[r, j] = p @ v[:, h], p @ v[:, h].abs(), torch.logsumexp(s, 0)
    return out, lse, mag, big


def check(torch, got, got_lse, ref, u, n, D):
    out, lse, mag, big = ref
    ds = ((D + 8) * 2.0 ** -23 * big)[..., None]
    tol = u * out.abs() + (u + 2 * ds + (n + 16) * 2.0 ** -23) * mag
    err = (got.cpu().double() - out).abs()
    assert bool((err <= tol).all()), f"out: worst {float((err / tol.clamp(min=1e-300)).max()):.3g} of the bound"
    if got_lse is not None:
        g = got_lse.cpu().double()
        none = torch.isinf(lse)
        assert bool((torch.isinf(g) == none).all()) and bool((g[none] < 0).all())
        tl = ds[..., 0] + (n + 16) * 2.0 ** -23 + 2.0 ** -22 * lse.abs()
        assert bool(((g - lse).abs() <= tl)[~none].all()), "lse"


U = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def make(torch, R, Hq, Hk, D, prefix_len, lens, pt, dtype="bfloat16", seed=0, q_std=2.0, poison=True, extra=3):
    """Pool, queries, prefix pages, tables and lengths; what lies behind the lengths is NaN and infinity."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt = getattr(torch, dtype)
    lens = np.asarray(lens, dtype=np.int32)
    npre = -(-prefix_len // pt)
    held = -(-lens // pt)
    pages = npre + int(held.sum()) + extra
    perm = rng.permutation(pages).astype(np.int32)
    cols = max(1, int(held.max()) if lens.size else 1)
    tables = np.full((R, cols), -1, dtype=np.int32)
    at = npre
    for r in range(R):
        tables[r, :held[r]] = perm[at:at + held[r]]
        at += held[r]
    pool = torch.randn((1, 2, pages, pt, Hk, D), generator=gen, device="cuda").to(dt)
    if poison:
        bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda").to(dt)
        fill = bad[torch.arange(Hk * D, device="cuda") % 3].view(Hk, D)
        pool[:, :, torch.from_numpy(perm[at:]).cuda().long()] = fill
        if prefix_len % pt:
            pool[:, :, int(perm[npre - 1]), prefix_len % pt:] = fill
        for r in range(R):
            if lens[r] % pt:
                pool[:, :, int(tables[r, held[r] - 1]), lens[r] % pt:] = fill
    q = (torch.randn((R, Hq, D), generator=gen, device="cuda") * q_std).to(dt)
    c = lambda a: torch.from_numpy(a).cuda()
    return pool, q, c(perm[:npre].copy()), c(tables), c(lens)


def run(torch, pool, q, prefix, prefix_len, tables, lens, scale=None, stream=None):
    from paper_2609_09800_amd import hbf
    kv = hbf.KvPages(pool)
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device="cuda")
    rc = kv.prefix_attention(0, q, out, prefix, prefix_len, tables, lens, lse=lse, scale=scale, stream=stream)
    assert rc == OK
    return kv, out, lse


CASES = [
    # rows, heads, kv heads, dim, prefix, own lengths, page
    (1, 8, 1, 128, 1, [0], 16), (1, 8, 1, 128, 0, [1], 16), (1, 1, 1, 64, 33, [31], 8), (2, 4, 4, 64, 0, [0, 0], 16),
    (3, 6, 2, 128, 0, [0, 5, 700], 16), (5, 16, 1, 64, 129, [0, 1, 15, 16, 17], 1), (2, 64, 2, 128, 1000, [40, 0], 7),
    (7, 6, 2, 64, 1003, [130, 0, 3, 24, 25, 48, 99], 24), (4, 8, 1, 128, 4096, [300, 1, 2, 128], 16),
    (16, 32, 4, 128, 777, list(range(0, 160, 10)), 64), (9, 16, 2, 64, 2000, [5] * 9, 16),
    (33, 8, 2, 128, 511, [1] * 33, 256), (64, 32, 4, 128, 300, [0] * 64, 16), (130, 4, 1, 64, 65, [2] * 130, 3),
    (1, 48, 1, 128, 640, [1000], 16), (2, 20, 1, 64, 0, [513, 64], 32), (1, 32, 4, 128, 20000, [1], 16),
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:5]) + f"-p{c[6]}")
def test_against_64_bits(torch, case, dtype):
    R, Hq, Hk, D, L, lens, pt = case
    say(f"attention {case} {dtype}")
    pool, q, prefix, tables, ln = make(torch, R, Hq, Hk, D, L, lens, pt, dtype, seed=R + L)
    kv, out, lse = run(torch, pool, q, prefix, L, tables, ln)
    assert kv.get_status() == OK
    ref = reference(torch, pool[0], q, prefix, L, tables, ln, D ** -0.5)
    check(torch, out, lse, ref, U[dtype], L + max(lens), D)


@pytest.mark.parametrize("scale,q_std", [(0.0, 1.0), (-0.3, 1.0), (0.5, 8.0), (1e-3, 0.1)])
def test_scales(torch, scale, q_std):
    """Flat, reversed and nearly one-hot softmaxes."""
    pool, q, prefix, tables, ln = make(torch, 4, 8, 2, 64, 200, [0, 10, 33, 100], 16, seed=3, q_std=q_std)
    kv, out, lse = run(torch, pool, q, prefix, 200, tables, ln, scale=scale)
    check(torch, out, lse, reference(torch, pool[0], q, prefix, 200, tables, ln, scale), U["bfloat16"], 300, 64)


def test_rising_scores(torch):
    """The running maximum moves at every step, by far more than the type's range of exp."""
    pool, q, prefix, tables, ln = make(torch, 3, 8, 1, 64, 1500, [700, 0, 90], 16, seed=4)
    ramp = torch.linspace(-30, 30, 1500, device="cuda")
    k = pool[0, 0, prefix.long()].view(-1, 64)
    k[:1500, 0] = ramp.bfloat16()
    pool[0, 0, prefix.long()] = k.view(-1, 16, 1, 64)
    q[:, :, 0] = 40.0
    for order in (prefix, prefix):
        kv, out, lse = run(torch, pool, q, order, 1500, tables, ln)
        check(torch, out, lse, reference(torch, pool[0], q, order, 1500, tables, ln, 0.125), U["bfloat16"], 2200, 64)
    k[:1500, 0] = -ramp.bfloat16()
    pool[0, 0, prefix.long()] = k.view(-1, 16, 1, 64)
    kv, out, lse = run(torch, pool, q, prefix, 1500, tables, ln)
    check(torch, out, lse, reference(torch, pool[0], q, prefix, 1500, tables, ln, 0.125), U["bfloat16"], 2200, 64)


def test_infinite_scores_in_one_part(torch):
    """Tokens whose score is -infinity weigh nothing, wherever the token axis is cut; a row that has only such
    tokens is NaN as the softmax of them is, and its sum's logarithm -infinity."""
    pool, q, prefix, tables, ln = make(torch, 2, 4, 1, 64, 1000, [40, 64], 16, seed=5)
    q[:, :, 0] = 1.0
    pages = prefix.long()
    k = pool[0, 0, pages].view(-1, 64)
    k[:600, 0] = -math.inf
    pool[0, 0, pages] = k.view(-1, 16, 1, 64)
    kv, out, lse = run(torch, pool, q, prefix, 1000, tables, ln)
    keep = pool.clone()
    kept = keep[0, 0, pages].view(-1, 64)
    kept[:600, 0] = -60000.0   # finite, and as good as infinite
    keep[0, 0, pages] = kept.view(-1, 16, 1, 64)
    ref = reference(torch, keep[0], q, prefix, 1000, tables, ln, 0.125)
    ref = (ref[0], ref[1], ref[2], torch.full_like(ref[3], 60.0))   # the finite scores' size
    check(torch, out, lse, ref, U["bfloat16"], 1100, 64)
    kv, out, lse = run(torch, pool, q, prefix, 600, torch.zeros_like(tables), torch.zeros_like(ln))
    assert bool(torch.isnan(out).all()) and bool((lse == -math.inf).all())


def test_nan_in_a_row_of_its_own_stays_there(torch):
    pool, q, prefix, tables, ln = make(torch, 3, 8, 2, 64, 100, [20, 20, 20], 16, seed=6)
    want = run(torch, pool, q, prefix, 100, tables, ln)[1]
    pool[0, 1, int(tables[1, 0]), 3] = math.nan
    q2 = q.clone()
    q2[2, 5, 7] = math.nan
    out = run(torch, pool, q2, prefix, 100, tables, ln)[1]
    assert torch.equal(out[0], want[0]) and bool(torch.isnan(out[1]).all())
    assert bool(torch.isnan(out[2, 5]).all()) and torch.equal(out[2, :5], want[2, :5])


def test_strides_and_layouts(torch):
    """Queries and outputs inside wider tensors, a table's columns behind the prefix, another layer of the pool."""
    from paper_2609_09800_amd import hbf
    pool, q, prefix, tables, ln = make(torch, 5, 8, 2, 64, 96, [0, 40, 17, 5, 80], 16, seed=7)
    want = run(torch, pool, q, prefix, 96, tables, ln)[1:]
    two = torch.randn((2, *pool.shape[1:]), device="cuda").bfloat16()
    two[1] = pool[0]
    wide = torch.full((5, 3, 8, 72), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 1, :, :64] = q
    out = torch.full((5, 8, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    table = torch.cat([prefix[None].expand(5, -1), tables], 1).contiguous()   # as a forked cache's rows look
    lse = torch.empty((5, 8), dtype=torch.float32, device="cuda")
    kv = hbf.KvPages(two)
    assert kv.prefix_attention(1, wide[:, 1, :, :64], out[:, :, 1], table[0, :6].contiguous(), 96, table[:, 6:], ln, lse=lse) == OK
    assert torch.equal(out[:, :, 1], want[0]) and torch.equal(lse, want[1])
    assert bool((out[:, :, 0] == 5.0).all())
    # without lse; without own tokens; prefix of zero length
    o2 = torch.empty_like(q)
    assert kv.prefix_attention(1, q, o2, prefix, 96, tables, ln) == OK and torch.equal(o2, want[0])
    assert kv.prefix_attention(1, q, o2, prefix, 96) == OK
    assert torch.equal(o2, run(torch, pool, q, prefix, 96, torch.zeros_like(tables), torch.zeros_like(ln))[1])
    assert kv.prefix_attention(1, q, o2, None, 0) == OK and not o2.any()
    assert kv.prefix_attention(1, q[:0], o2[:0], prefix, 96) == OK
    assert kv.get_status() == OK


def test_rows_do_not_meet(torch):
    """A row's result does not depend on its place in the batch beyond rounding, and repeats bit for bit."""
    pool, q, prefix, tables, ln = make(torch, 40, 8, 2, 128, 700, [int(x) for x in np.arange(40) * 7 % 90], 16, seed=8)
    a = run(torch, pool, q, prefix, 700, tables, ln)
    b = run(torch, pool, q, prefix, 700, tables, ln)
    assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])


def test_offsets_past_32_bits(torch):
    """Pages behind 2^32 bytes of a 9 GiB pool."""
    from paper_2609_09800_amd import hbf
    pages, pt = 9000, 1024
    pool = torch.zeros((1, 2, pages, pt, 4, 64), dtype=torch.bfloat16, device="cuda")
    small, q, prefix, tables, ln = make(torch, 2, 8, 4, 64, 1500, [100, 1030], pt, seed=9)
    move = torch.arange(small.shape[2], device="cuda") + pages - small.shape[2]
    pool[:, :, move] = small
    up = lambda t: torch.where(t >= 0, move[t.clamp(min=0).long()].int(), -1)
    want = run(torch, small, q, prefix, 1500, tables, ln)[1]
    got = run(torch, pool, q, up(prefix), 1500, up(tables), ln)[1]
    assert torch.equal(got, want)


@pytest.mark.parametrize("what", ["length", "negative", "page", "page_low", "prefix"])
def test_bad_entries_fail_closed(torch, what):
    """A length or page out of range: that row is NaN (all of them for the prefix), the others are right."""
    pool, q, prefix, tables, ln = make(torch, 4, 8, 2, 64, 90, [20, 30, 16, 5], 16, seed=10)
    want = run(torch, pool, q, prefix, 90, tables, ln)[1]
    if what == "length":
        ln[1] = tables.shape[1] * 16 + 1
    elif what == "negative":
        ln[1] = -1
    elif what == "page":
        tables[1, 1] = pool.shape[2]
    elif what == "page_low":
        tables[1, 0] = -1
    else:
        prefix[3] = 1 << 30
    kv, out, lse = run(torch, pool, q, prefix, 90, tables, ln)
    assert kv.get_status() == EINVAL and kv.get_status() == OK
    bad = torch.tensor([True] * 4 if what == "prefix" else [False, True, False, False], device="cuda")
    assert bool(torch.isnan(out[bad]).all()) and bool(torch.isnan(lse[bad]).all())
    assert torch.equal(out[~bad], want[~bad])


def test_refusals(torch):
    from paper_2609_09800_amd import hbf
    pool, q, prefix, tables, ln = make(torch, 4, 8, 2, 64, 90, [20, 30, 16, 5], 16, seed=11)
    kv, out, lse = run(torch, pool, q, prefix, 90, tables, ln)
    for args in ((1, q, out, prefix, 90, tables, ln), (0, q.float(), out, prefix, 90, tables, ln),
                 (0, q, out[:3], prefix, 90, tables, ln), (0, q, out, prefix[:2], 90, tables, ln),
                 (0, q, out, prefix, 90, tables, None), (0, q, out, prefix, 90, tables[:3], ln),
                 (0, q, out, prefix, 90, tables.long(), ln), (0, q, out, prefix, 90, tables, ln.long()),
                 (0, q.cpu(), out, prefix, 90, tables, ln), (0, q, out[:1].expand(4, -1, -1), prefix, 90, tables, ln),
                 (0, q.transpose(1, 2).contiguous().transpose(1, 2), out, prefix, 90, tables, ln),
                 (0, q, out, prefix.long(), 90, tables, ln), (0, q[..., :32], out[..., :32], prefix, 90, tables, ln)):
        with pytest.raises(hbf.HbfError):
            kv.prefix_attention(*args)
    assert kv.prefix_attention(0, q[:, :7], out[:, :7], prefix, 90, tables, ln) == EINVAL     # 7 heads over 2
    assert kv.prefix_attention(0, q, out, prefix, -1, tables, ln) == EINVAL
    assert kv.prefix_attention(0, q, out, prefix, 90, tables, ln, scale=math.nan) == EINVAL
    odd = torch.zeros((1, 2, 4, 16, 2, 96), dtype=torch.bfloat16, device="cuda")              # head_dim 96
    q96 = torch.zeros((1, 2, 96), dtype=torch.bfloat16, device="cuda")
    assert hbf.KvPages(odd).prefix_attention(0, q96, q96.clone(), prefix, 16) == EINVAL


def test_another_stream_and_graph(torch):
    from paper_2609_09800_amd import hbf
    pool, q, prefix, tables, ln = make(torch, 6, 8, 2, 128, 900, [20, 0, 130, 5, 64, 33], 16, seed=12)
    want = run(torch, pool, q, prefix, 900, tables, ln)[1]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    kv, out, _ = run(torch, pool, q, prefix, 900, tables, ln, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    q2 = q.clone()
    out.zero_()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert kv.prefix_attention(0, q2, out, prefix, 900, tables, ln) == OK
    for i in range(4):
        q2.copy_(q * (i + 1) / 2)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, run(torch, pool, q2, prefix, 900, tables, ln)[1])


# rows, heads, kv heads, dim, prefix, own lengths, page: 1, 2 and 4 queries for each part of the joining workgroup, as
# many parts as it takes and one more, a head with rows that have nothing, more heads than control words
JOINED = [(1, 8, 1, 128, 3000, [20], 16), (1, 8, 2, 128, 4096, [300], 16), (1, 8, 2, 64, 24 * 256, [0], 16),
          (2, 16, 1, 128, 700, [64, 0], 8), (2, 16, 2, 64, 1500, [0, 200], 16), (4, 32, 4, 128, 600, [9, 0, 90, 1], 16),
          (4, 7, 1, 128, 130, [0, 0, 0, 0], 16), (5, 6, 1, 64, 0, [0, 0, 3, 0, 0], 16), (1, 65, 65, 64, 40, [5], 8)]


@pytest.mark.parametrize("case", JOINED, ids=lambda c: "-".join(str(x) for x in c[:5]))
def test_joined_in_the_launch_or_after_it(torch, case):
    """Both forms, in turn on one object, from scratch that held anything."""
    R, Hq, Hk, D, L, lens, pt = case
    say(f"attention joined {case}")
    pool, q, prefix, tables, ln = make(torch, R, Hq, Hk, D, L, lens, pt, seed=21)
    kv, out, lse = run(torch, pool, q, prefix, L, tables, ln)
    ref = reference(torch, pool[0], q, prefix, L, tables, ln, D ** -0.5)
    status, words = kv._attn_at
    for with_words in (True, False, True, True):
        kv._attn_ws._t.fill_(255)
        out.fill_(7.0)
        kv._attn_at = (status, words if with_words else None)
        assert kv.prefix_attention(0, q, out, prefix, L, tables, ln, lse=lse) == OK
        check(torch, out, lse, ref, U["bfloat16"], L + max(lens), D)
        assert not bool(kv._attn_ctl.any())
    assert kv.get_status() == OK
