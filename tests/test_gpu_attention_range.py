"""Attention over the whole range of scores and probabilities, in 64 bits.

Scores here are exact in 32 bits, so that only what follows them is bounded:
with u the 16-bit type's unit roundoff,
    |o - o64| <= u |o| + (u + 2 ds + (n + 16) 2^-23) sum p |v| + cut,  ds = (D + 8) 2^-23 max |s|,
where ds bounds the rounding of the exponent (s - m) scale log2 e of scores that
differ by a few, and is 0 where they are equal or too far apart to count; cut is
what the type's range leaves out.
"""
import math

import pytest

from test_gpu_kv_attention import EINVAL, OK, U, make, reference, run, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    from paper_2609_09800_amd import hbf
    hbf.load_library()
    return t


# rows, heads, kv heads, prefix, own lengths: joined in the launch; by one of its own; many queries
SHAPES = [(1, 8, 1, 300, [33]), (2, 16, 2, 4000, [700, 0]), (40, 8, 2, 1000, [0, 1, 17, 130] * 10)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
@pytest.mark.parametrize("dtype,q_value,unit", [
    ("bfloat16", 2.0 ** 10, 2.0 ** 12), ("bfloat16", 2.0 ** 20, 2.0 ** 20), ("bfloat16", 2.0 ** 50, 2.0 ** 60),
    ("float16", 2.0 ** 10, 2.0 ** 8), ("float16", 2.0 ** 15, 2.0 ** 12)])
@pytest.mark.parametrize("low,high", [(-7, 7), (-15, -3)])
def test_scores_of_any_size(torch, dtype, q_value, unit, low, high, shape):
    """Scores of up to 2^118, far past where one step of a float is more than the range of exp: the highest tokens,
    and as many as tie, share the row."""
    R, Hq, Hk, L, lens = shape
    say(f"attention scores {dtype} {q_value} {unit} {low} {high} {shape}")
    pool, q, prefix, tables, ln = make(torch, R, Hq, Hk, 64, L, lens, 16, dtype, seed=31)
    gen = torch.Generator(device="cuda").manual_seed(32)
    keys = torch.randint(low, high + 1, pool.shape[2:5], generator=gen, device="cuda")
    keep = torch.isfinite(pool[0, 0])   # (what lies behind the lengths stays NaN and infinity)
    pool[0, 0] = torch.where(keep, (keys[..., None] * unit).to(pool.dtype), pool[0, 0])
    q[:] = q_value
    kv, out, lse = run(torch, pool, q, prefix, L, tables, ln, scale=0.125)
    assert kv.get_status() == OK
    want, want_lse, mag, _ = reference(torch, pool[0], q, prefix, L, tables, ln, 0.125)
    u, n = U[dtype], L + max(lens)
    err = (out.cpu().double() - want).abs()
    assert bool((err <= u * want.abs() + (u + (n + 16) * 2.0 ** -23) * mag).all())
    assert bool(((lse.cpu().double() - want_lse).abs() <= (n + 16) * 2.0 ** -23 + 2.0 ** -22 * want_lse.abs()).all())


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("every", [32, 64, 4096])
@pytest.mark.parametrize("gap", [9.0, 14.0, 17.0, 17.5, 19.0, 21.5, 24.0])
def test_many_small_probabilities(torch, gap, every, dtype):
    """Tokens of no value take nearly all of the weight, and the others, each e^-gap of it, make the result.  What is
    smaller than the type's steps is rounded to one: per token at most 2^-32 of the largest probability."""
    for R, Hq, Hk, L, lens in ((1, 8, 1, 4099, [77]), (33, 8, 2, 4099, [0, 64, 300] * 11)):
        say(f"attention small probabilities {gap} {every} {dtype} {R}")
        pool, q, prefix, tables, ln = make(torch, R, Hq, Hk, 64, L, lens, 16, dtype, seed=33)
        seen = torch.isfinite(pool[0, 0])
        value = torch.rand(pool.shape[2:], generator=torch.Generator(device="cuda").manual_seed(34), device="cuda") * 500 + 500
        pool[0, 0] = torch.where(seen, torch.zeros_like(pool[0, 0]), pool[0, 0])
        pool[0, 1] = torch.where(seen, value.to(pool.dtype), pool[0, 1])
        big = torch.arange(0, L, every, device="cuda")
        page, token = prefix[big // 16].long(), big % 16
        pool[0, 0, page, token, :, 0] = gap
        pool[0, 1, page, token] = 0.0
        q.zero_()
        q[:, :, 0] = 1.0
        kv, out, lse = run(torch, pool, q, prefix, L, tables, ln, scale=1.0)
        assert kv.get_status() == OK
        want, want_lse, mag, _ = reference(torch, pool[0], q, prefix, L, tables, ln, 1.0)
        n, u, ds = L + max(lens), U[dtype], 72 * 2.0 ** -23 * gap
        cut = 2.0 ** -32 * n * 1000 * torch.exp(gap - want_lse)[..., None] + 2.0 ** -25   # (and a half's own last step)
        err = (out.cpu().double() - want).abs()
        assert bool((err <= u * want.abs() + (u + 2 * ds + (n + 16) * 2.0 ** -23) * mag + cut).all())
        assert bool(((lse.cpu().double() - want_lse).abs() <= ds + (n + 16) * 2.0 ** -23 + 2.0 ** -22 * want_lse.abs()).all())


def test_scales_at_the_type_s_ends(torch):
    """Past them: refused.  At them: the highest token alone; all alike."""
    pool, q, prefix, tables, ln = make(torch, 2, 8, 2, 64, 90, [20, 30], 16, seed=35)
    kv, out, lse = run(torch, pool, q, prefix, 90, tables, ln)
    for scale in (1e39, -1e300, math.inf):
        assert kv.prefix_attention(0, q, out, prefix, 90, tables, ln, scale=scale) == EINVAL
    for scale in (3.4e38, 1e-44):
        kv, out, lse = run(torch, pool, q, prefix, 90, tables, ln, scale=scale)
        want = reference(torch, pool[0], q, prefix, 90, tables, ln, scale)[0]
        assert bool(((out.cpu().double() - want).abs() <= U["bfloat16"] * (want.abs() + 4)).all())
