"""The mixture-of-experts layer against its definition in 64 bits.

Tolerance, per element, from the formulas (u: the 16-bit type's unit roundoff,
e = 2^-23 twice the fp32 one): sums of n products carry n e of the sum of their
magnitudes, so
    dg, du = (H + 8) e sum |w||x|,   dh = (1.1 dg + 8 e |silu|) |up| + (|silu| + dg) du + (u^2 + 8 e) |h|,
    dw = (2 (H + 8) e sum |r||x| + (E + 16) e) w,
    |y - y64| <= u |y| + sum_j [ dw_j |d.h| + w_j (sum |d| dh + (F + 8) e sum |d||h|) ] + (k + 2) e sum |w_j d.h|.
The j-th choice must be the j-th largest logit's, or one within both logits'
error of it; where logits are exact, the very one.
"""
import math
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

OK, EINVAL, ENOWORKSPACE = 0, -1, -4
U = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
EPS = 2.0 ** -23


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


def make(torch, T, E, H, F, dtype, seed=0, std=1.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = getattr(torch, dtype)
    r = lambda shape, s: (torch.randn(shape, generator=gen, device="cuda") * s).to(dt)
    return r((T, H), std), r((E, H), 1 / math.sqrt(H)), r((E, 2 * F, H), 1 / math.sqrt(H)), r((E, H, F), 1 / math.sqrt(F))


def reference(torch, x, gate_up, down, topk, u, router=None, ids=None, weights=None, renorm=True):
    """y, ids, weights and the bounds of y and weights, in 64 bits."""
    xd = x.double()
    T, H = x.shape
    E, F2, _ = gate_up.shape
    F = F2 // 2
    if router is not None:
        logits = (xd @ router.double().t()).cpu().numpy()
        mag = (xd.abs() @ router.double().abs().t()).cpu().numpy()
        best = np.stack([np.lexsort((np.arange(E), -l))[:topk] for l in logits])
        ids = ids.cpu().numpy()   # what the layer chose
        bound = 2 * (H + 8) * EPS * mag.max(1, keepdims=True)
        short = np.take_along_axis(logits, best, 1) - np.take_along_axis(logits, ids, 1)
        assert ((ids == best) | (np.abs(short) <= bound)).all(), "choices"
        assert all(len(set(r)) == topk for r in ids.tolist())
        p = np.exp(logits - logits.max(1, keepdims=True))
        w = np.take_along_axis(p, ids, 1) / (np.take_along_axis(p, ids, 1) if renorm else p).sum(1, keepdims=True)
        rel = bound + (E + 16) * EPS
    else:
        ids, w = ids.cpu().numpy(), weights.double().cpu().numpy()
        rel = np.zeros((T, 1))
    y = torch.zeros((T, H), dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(y)
    mags = torch.zeros_like(y)
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if not t.size:
            continue
        td = torch.from_numpy(t).cuda()
        wj = torch.from_numpy(w[t, j]).cuda()[:, None]
        rl = torch.from_numpy(np.broadcast_to(rel, (T, topk))[t, j].copy()).cuda()[:, None]
        wt = gate_up[e].double().t().contiguous()
        both = xd[td] @ wt
        d_both = (H + 8) * EPS * (xd[td].abs() @ wt.abs())
        g, up, dg, du = both[:, :F], both[:, F:], d_both[:, :F], d_both[:, F:]
        silu = g * torch.sigmoid(g)
        h = silu * up
        dh = (1.1 * dg + 8 * EPS * silu.abs()) * up.abs() + (silu.abs() + 1.1 * dg) * du + (u * u + 8 * EPS) * h.abs()
        dt = down[e].double().t().contiguous()
        o = h @ dt
        err = dh @ dt.abs() + (F + 8) * EPS * (h.abs() @ dt.abs())
        y.index_add_(0, td, wj * o)
        tol.index_add_(0, td, wj * err + rl * wj * o.abs())
        mags.index_add_(0, td, (wj * o).abs())
    return y, ids, w, u * y.abs() + 1.01 * tol + (topk + 2) * EPS * mags + 1e-30, rel


def run(torch, x, gate_up, down, topk, router=None, ids=None, weights=None, renorm=True, stream=None, layer=None):
    from paper_2609_09800_amd import hbf
    T = x.shape[0]
    layer = layer or hbf.MoeLayer(gate_up, down, topk, router=router, renormalize=renorm, max_tokens=max(T, 1))
    y = torch.full_like(x, 7.0)
    if router is not None:
        ids = torch.full((T, topk), -7, dtype=torch.int32, device="cuda")
        weights = torch.full((T, topk), -7.0, dtype=torch.float32, device="cuda")
    assert layer.forward(x, y, ids, weights, stream=stream) == OK
    return layer, y, ids, weights


def check(torch, got, ref, ids=None, weights=None):
    y, rids, rw, tol, rel = ref
    err = (got.double() - y).abs()
    assert bool((err <= tol).all()), f"y: worst {float((err / tol).max()):.3g} of the bound"
    if ids is not None:
        assert np.array_equal(ids.cpu().numpy(), rids)
        assert (np.abs(weights.double().cpu().numpy() - rw) <= rel * rw + 1e-30).all()


CASES = [
    # tokens, experts, topk, hidden, ffn
    (1, 128, 8, 2048, 768), (64, 128, 8, 2048, 768), (1, 1, 1, 8, 8), (3, 2, 2, 16, 24), (5, 20, 3, 328, 104),
    (17, 8, 1, 512, 64), (2, 64, 6, 1024, 136), (33, 100, 5, 200, 56), (128, 16, 4, 264, 40), (128, 8, 8, 128, 1032),
    (1, 1024, 32, 64, 16), (40, 300, 7, 256, 32), (16, 4, 2, 4104, 72), (7, 5, 5, 72, 2056),
]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_layer_against_64_bits(torch, case, dtype):
    T, E, k, H, F = case
    say(f"moe {case} {dtype}")
    x, router, gate_up, down = make(torch, T, E, H, F, dtype, seed=T + E)
    layer, y, ids, w = run(torch, x, gate_up, down, k, router=router)
    check(torch, y, reference(torch, x, gate_up, down, k, U[dtype], router=router, ids=ids), ids, w)
    assert layer.get_status() == OK


# few token tiles: whole passes over the inner axis, part of one, several; rows that end inside a workgroup
@pytest.mark.parametrize("case", [(1, 16, 8, 4096, 768), (2, 6, 3, 4104, 1544), (3, 9, 5, 24, 264), (16, 2, 1, 40, 768),
                                  (1, 8, 8, 4096, 256)], ids=lambda c: "-".join(map(str, c)))
def test_few_token_tiles(torch, case):
    T, E, k, H, F = case
    say(f"moe few tiles {case}")
    x, router, gate_up, down = make(torch, T, E, H, F, "bfloat16", seed=T + H)
    layer, y, ids, w = run(torch, x, gate_up, down, k, router=router)
    check(torch, y, reference(torch, x, gate_up, down, k, U["bfloat16"], router=router, ids=ids), ids, w)
    assert layer.get_status() == OK


def test_weights_over_all_experts(torch):
    x, router, gate_up, down = make(torch, 9, 12, 64, 32, "bfloat16", seed=2)
    _, y, ids, w = run(torch, x, gate_up, down, 3, router=router, renorm=False)
    check(torch, y, reference(torch, x, gate_up, down, 3, U["bfloat16"], router=router, ids=ids, renorm=False), ids, w)


@pytest.mark.parametrize("E,k", [(16, 4), (70, 9), (200, 20), (700, 32)])
def test_ties_go_to_the_lowest_index(torch, E, k):
    """Logits that are small whole numbers, many equal (0 and -0 among them)."""
    T, H = 20, 16
    x, router, gate_up, down = make(torch, T, E, H, 8, "bfloat16", seed=3)
    rng = np.random.default_rng(E)
    x = torch.from_numpy(rng.integers(-1, 2, (T, H)).astype(np.float32)).cuda().bfloat16()
    router = torch.from_numpy(rng.integers(-1, 2, (E, H)).astype(np.float32)).cuda().bfloat16()
    x[0] = 0
    x[1] = -0.0
    logits = (x.double() @ router.double().t()).cpu().numpy()
    best = np.stack([np.lexsort((np.arange(E), -l))[:k] for l in logits])
    _, y, ids, w = run(torch, x, gate_up, down, k, router=router)
    check(torch, y, reference(torch, x, gate_up, down, k, U["bfloat16"], router=router, ids=ids), ids, w)
    assert np.array_equal(ids.cpu().numpy(), best)


def test_all_tokens_one_expert(torch):
    """The most uneven choice: more tokens of one expert than a tile holds, and tokens in common."""
    T, E, k = 100, 6, 2
    x, router, gate_up, down = make(torch, T, E, 264, 72, "bfloat16", seed=4)
    router = torch.zeros_like(router)
    router[4], router[2] = x.float().mean(0).bfloat16(), x.float().mean(0).bfloat16()
    x = (x.float() + 3 * x.float().mean(0).sign()).bfloat16()
    _, y, ids, w = run(torch, x, gate_up, down, k, router=router)
    check(torch, y, reference(torch, x, gate_up, down, k, U["bfloat16"], router=router, ids=ids), ids, w)


def given(torch, T, k, E, seed=5):
    rng = np.random.default_rng(seed)
    ids = rng.integers(-1, E, (T, k)).astype(np.int32)
    w = rng.standard_normal((T, k)).astype(np.float32)
    w[ids < 0] = np.nan   # an unused choice's weight is not looked at
    return torch.from_numpy(ids).cuda(), torch.from_numpy(w).cuda()


@pytest.mark.parametrize("T,E,k", [(1, 4, 2), (20, 6, 5), (64, 3, 32), (128, 40, 16)])
def test_given_choices(torch, T, E, k):
    """Choices of the caller's: none (-1), one expert twice, weights of any sign; more choices than experts."""
    x, _, gate_up, down = make(torch, T, E, 136, 40, "bfloat16", seed=6)
    ids, w = given(torch, T, k, E)
    ids[0] = -1
    if T > 1:
        ids[1] = 2
        w[1] = 0.5
    before = ids.clone(), w.clone()
    layer, y, _, _ = run(torch, x, gate_up, down, k, ids=ids, weights=w)
    ref = reference(torch, x, gate_up, down, k, U["bfloat16"], ids=ids, weights=w.nan_to_num())
    mags = ref[3]
    # weights of both signs: the bound's terms take their size
    pos = reference(torch, x, gate_up, down, k, U["bfloat16"], ids=ids, weights=w.nan_to_num().abs())
    err = (y.double() - ref[0]).abs()
    assert bool((err <= U["bfloat16"] * ref[0].abs() + pos[3]).all())
    assert not y[0].any() and layer.get_status() == OK
    assert torch.equal(ids, before[0]) and torch.equal(w.nan_to_num(), before[1].nan_to_num())


def test_no_choice_at_all(torch):
    x, _, gate_up, down = make(torch, 4, 3, 64, 16, "float16", seed=7)
    ids = torch.full((4, 2), -1, dtype=torch.int32, device="cuda")
    _, y, _, _ = run(torch, x, gate_up, down, 2, ids=ids, weights=torch.full((4, 2), math.nan, device="cuda"))
    assert not y.any()


def test_ids_out_of_range(torch):
    x, _, gate_up, down = make(torch, 4, 3, 64, 16, "bfloat16", seed=8)
    ids = torch.tensor([[0, 1], [2, 3], [-2, 0], [1, 2**31 - 1]], dtype=torch.int32, device="cuda")
    w = torch.ones((4, 2), device="cuda")
    layer, y, _, _ = run(torch, x, gate_up, down, 2, ids=ids, weights=w)
    assert layer.get_status() == EINVAL and layer.get_status() == OK
    ok = torch.where((ids >= 0) & (ids < 3), ids, -1)
    assert torch.equal(y, run(torch, x, gate_up, down, 2, ids=ok, weights=w)[1])


def test_nan_and_infinity_stay_in_their_token(torch):
    x, router, gate_up, down = make(torch, 6, 8, 72, 24, "bfloat16", seed=9)
    want = run(torch, x, gate_up, down, 2, router=router)
    x2 = x.clone()
    x2[1, 5] = math.nan
    x2[4, 0] = math.inf
    got = run(torch, x2, gate_up, down, 2, router=router)
    for t in (0, 2, 3, 5):
        assert torch.equal(got[1][t], want[1][t]) and torch.equal(got[2][t], want[2][t])
    assert bool(torch.isnan(got[1][1]).all())
    assert bool(((got[2] >= 0) & (got[2] < 8)).all()) and all(len(set(r)) == 2 for r in got[2].tolist())


def test_large_activations(torch):
    """Gates far out on both sides; h past the fp16 range would be infinite there, stays finite in bfloat16."""
    x, router, gate_up, down = make(torch, 8, 4, 64, 32, "bfloat16", seed=10, std=300.0)
    ids, w = given(torch, 8, 2, 4)
    ids = ids.clamp(min=0)
    w = w.nan_to_num().abs()
    _, y, _, _ = run(torch, x, gate_up, down, 2, ids=ids, weights=w)
    check(torch, y, reference(torch, x, gate_up, down, 2, U["bfloat16"], ids=ids, weights=w))


def test_one_buffer_of_experts_and_strided_rows(torch):
    """Expert after expert in one buffer (gate, up, down), tokens inside wider rows."""
    T, E, k, H, F = 11, 5, 2, 128, 48
    x, router, gate_up, down = make(torch, T, E, H, F, "bfloat16", seed=11)
    want = run(torch, x, gate_up, down, k, router=router)
    buf = torch.cat([gate_up.reshape(E, -1), down.reshape(E, -1), torch.zeros((E, 64), dtype=x.dtype, device="cuda")], 1)
    gu = buf[:, :2 * F * H].view(E, 2 * F, H)
    dn = buf[:, 2 * F * H:3 * F * H].view(E, H, F)
    wide = torch.full((T, H + 24), 9.0, dtype=x.dtype, device="cuda")
    wide[:, 8:8 + H] = x
    out = torch.full((T, H + 40), 9.0, dtype=x.dtype, device="cuda")
    from paper_2609_09800_amd import hbf
    layer = hbf.MoeLayer(gu, dn, k, router=router)
    ids = torch.empty((T, k), dtype=torch.int32, device="cuda")
    w = torch.empty((T, k), dtype=torch.float32, device="cuda")
    assert layer.forward(wide[:, 8:8 + H], out[:, 16:16 + H], ids, w) == OK
    assert torch.equal(out[:, 16:16 + H], want[1]) and torch.equal(ids, want[2]) and torch.equal(w, want[3])
    assert bool((out[:, :16] == 9.0).all()) and bool((out[:, 16 + H:] == 9.0).all())
    # calls of fewer tokens on the same object, and none
    assert layer.forward(x[:1], out[:1, 16:16 + H], ids[:1], w[:1]) == OK
    assert torch.equal(ids[0], want[2][0])
    assert layer.forward(x[:0], out[:0, :H], ids[:0], w[:0]) == OK


def test_repeats_bit_for_bit(torch):
    x, router, gate_up, down = make(torch, 50, 32, 512, 128, "bfloat16", seed=12)
    a = run(torch, x, gate_up, down, 4, router=router)
    b = run(torch, x, gate_up, down, 4, router=router, layer=a[0])
    assert torch.equal(a[1], b[1])


def test_refusals(torch):
    from paper_2609_09800_amd import hbf
    x, router, gate_up, down = make(torch, 4, 6, 64, 16, "bfloat16", seed=13)
    layer, y, ids, w = run(torch, x, gate_up, down, 2, router=router)
    for args in ((x.float(), y, ids, w), (x, y[:3], ids, w), (x[:, :56], y, ids, w), (x, y, ids.long(), w),
                 (x, y, ids[:, :1], w), (x, y, ids, w.double()), (x.cpu(), y, ids, w), (x.t(), y, ids, w),
                 (x, y[:1].expand(4, -1), ids, w)):
        with pytest.raises(hbf.HbfError):
            layer.forward(*args)
    many = torch.zeros((5, 64), dtype=x.dtype, device="cuda")
    i5, w5 = torch.zeros((5, 2), dtype=torch.int32, device="cuda"), torch.zeros((5, 2), device="cuda")
    assert layer.forward(many, many.clone(), i5, w5) == ENOWORKSPACE   # made for 4 tokens
    for bad in (dict(topk=7), dict(topk=0), dict(topk=33), dict(max_tokens=129), dict(max_tokens=-1)):
        with pytest.raises(hbf.HbfError):
            hbf.MoeLayer(gate_up, down, **{"topk": 2, "router": router, **bad})
    for args in ((gate_up.float(), down.float()), (gate_up, down.half()), (gate_up, down[:, :, :8]),
                 (gate_up[:, :31], down), (gate_up.transpose(1, 2), down), (gate_up, down[:5])):
        with pytest.raises(hbf.HbfError):
            hbf.MoeLayer(*args, 2)
    with pytest.raises(hbf.HbfError):
        hbf.MoeLayer(gate_up, down, 2, router=router[:5])
    with pytest.raises(hbf.HbfError):   # hidden 60 is no multiple of 8
        hbf.MoeLayer(gate_up[:, :, :60].contiguous(), down[:, :60].contiguous(), 2)


def test_another_stream_and_graph(torch):
    x, router, gate_up, down = make(torch, 8, 16, 256, 64, "bfloat16", seed=14)
    want = run(torch, x, gate_up, down, 4, router=router)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    layer, y, ids, w = run(torch, x, gate_up, down, 4, router=router, stream=s)
    s.synchronize()
    assert torch.equal(y, want[1])
    x2 = x.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert layer.forward(x2, y, ids, w) == OK
    for i in range(4):
        x2.copy_(x * (0.5 + i))
        g.replay()
        torch.cuda.synchronize()
        e = run(torch, x2, gate_up, down, 4, router=router)
        assert torch.equal(y, e[1]) and torch.equal(ids, e[2]) and torch.equal(w, e[3])
