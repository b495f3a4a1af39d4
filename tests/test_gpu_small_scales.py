"""Attention with small scales over large scores: softmaxes as uneven, or as even, as
the product of both says.  Scores are exact in 32 bits, and products with the scale
too but for the scale's own rounding with log2 e, so that of the bounds of the
tests named below only what follows the scores is left."""
import pytest

from test_gpu_attention_range import SHAPES as PREFIX_SHAPES
from test_gpu_chunk_attention import IDS, OK, SHAPES, U, batch, say, torch  # noqa: F401
from test_gpu_kv_attention import make, reference, run

pytestmark = pytest.mark.gpu

# q, K in multiples of, scale: scores of up to 448 and 112 steps of 2^110; probabilities of every size, and all alike
SCALES = [(2.0 ** 50, 2.0 ** 60, 2.0 ** -117), (2.0 ** 50, 2.0 ** 60, -(2.0 ** -118)), (2.0 ** 50, 2.0 ** 60, 0.0),
          (2.0 ** 50, 2.0 ** 60, 2.0 ** -140), (2.0 ** 20, 2.0 ** 76, 2.0 ** -103)]


@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
@pytest.mark.parametrize("q_value,unit,scale", SCALES)
def test_chunks(torch, q_value, unit, scale, shape):   # noqa: F811
    say(f"attention small scale {scale} {shape}")
    b = batch(torch, shape, seed=51)
    keys = torch.randint(-7, 8, b.pool.shape[2:5], generator=torch.Generator(device="cuda").manual_seed(52), device="cuda")
    keep = torch.isfinite(b.pool[0, 0])   # (what lies behind the lengths stays NaN and infinity)
    b.pool[0, 0] = torch.where(keep, (keys[..., None] * unit).to(b.pool.dtype), b.pool[0, 0])
    b.q[:] = q_value
    w = b.weights.clone()
    out, lse = b.run(scale=scale, weights=w)
    assert b.kv.get_status() == OK
    ref = list(b.reference(scale=scale, weights=b.weights))
    n = max(b.lens) + 32
    ref[3] = torch.zeros_like(ref[3])
    ref[5] = b.reference(scale=0.0, weights=b.weights)[5] + n * 2.0 ** -23 * ref[4]   # (every p at most 1)
    b.check(out, lse, ref, w)


@pytest.mark.parametrize("shape", PREFIX_SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
@pytest.mark.parametrize("q_value,unit,scale", SCALES)
def test_prefix(torch, q_value, unit, scale, shape):   # noqa: F811
    R, Hq, Hk, L, lens = shape
    say(f"prefix attention small scale {scale} {shape}")
    pool, q, prefix, tables, ln = make(torch, R, Hq, Hk, 64, L, lens, 16, "bfloat16", seed=53)
    keys = torch.randint(-7, 8, pool.shape[2:5], generator=torch.Generator(device="cuda").manual_seed(54), device="cuda")
    pool[0, 0] = torch.where(torch.isfinite(pool[0, 0]), (keys[..., None] * unit).to(pool.dtype), pool[0, 0])
    q[:] = q_value
    kv, out, lse = run(torch, pool, q, prefix, L, tables, ln, scale=scale)
    assert kv.get_status() == OK
    want, want_lse, mag, _ = reference(torch, pool[0], q, prefix, L, tables, ln, scale)
    u, n = U["bfloat16"], L + max(lens)
    err = (out.cpu().double() - want).abs()
    assert bool((err <= u * want.abs() + (u + (n + 16) * 2.0 ** -23) * mag).all())
    assert bool(((lse.cpu().double() - want_lse).abs() <= (n + 16) * 2.0 ** -23 + 2.0 ** -22 * want_lse.abs()).all())
