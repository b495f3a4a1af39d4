"""Weights that hold no token: as ones that hold too few.  Rows and sequences of a length are in error, empty ones are not."""
import pytest

from test_gpu_chunk_attention import EINVAL, OK, Batch, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new,lens,cols", [([1, 1, 0], [40, 0, 0], 0), ([1, 70, 1], [40, 90, 0], 1200)])
def test_attention(torch, new, lens, cols):   # noqa: F811
    say(f"weights of no tokens {lens}")
    b = Batch(torch, 16, 4, 64, new, lens, 16, cols=cols, seed=61)
    w = torch.zeros((b.weights.shape[0], 4, 0), device="cuda")
    out, lse = b.run(weights=w)
    assert b.kv.get_status() == EINVAL
    for s0, n, L in zip(b.starts, b.new, b.lens):
        if n:
            assert bool(torch.isnan(out[s0:s0 + n]).all()) if L else bool((out[s0:s0 + n] == 0).all())
    b.dev["lens"].zero_()
    out, lse = b.run(weights=w)
    assert b.kv.get_status() == OK and bool((out[:sum(new)] == 0).all())


def test_evict(torch):   # noqa: F811
    b = Batch(torch, 4, 2, 64, [0, 0], [0, 40], 16, seed=62)
    i32 = dict(dtype=torch.int32, device="cuda")
    for out in (None, torch.zeros((1, 3, 2, 0), device="cuda")):
        say(f"evict by weights of no tokens {out is not None}")
        for i, status in ((0, OK), (1, EINVAL)):   # an empty sequence, one of 40 tokens
            kept = torch.full((1, 1, 2, 5), 7, **i32)
            pool = b.pool.clone()
            assert b.kv.evict(b.dev["slots"][i:i + 1], torch.full((1,), 5, **i32), torch.zeros((1, 3, 2, 0), device="cuda"), kept,
                              weights_out=out) == OK
            assert b.kv.get_status() == status
            assert int(b.dev["lens"][int(b.slots[1])]) == 40 and torch.equal(pool.view(torch.int16), b.pool.view(torch.int16))
            if status == OK:
                assert bool((kept == -1).all())
