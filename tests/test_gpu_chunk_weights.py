"""What accumulated weights take from a query whose sums are not finite: it reaches
the tokens that the query sees, and no other.  By every way that weights are added
up: from scores that attention left (a row one tile of 16 queries, or several), from
K again for many queries, and for few."""
import math

import pytest

from test_gpu_chunk_attention import OK, Batch, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu

# heads, kv heads, dim, new tokens, lengths, page, extra columns; scores kept: in tiles of one a row, of several; from K
# again: tiles of 256, tiles of 16 and many queries, few of them beside tables of millions of tokens
WAYS = [(8, 2, 64, [1, 1, 2], [40, 300, 9], 16, 0), (8, 2, 128, [30, 1], [200, 77], 16, 0),
        (16, 4, 128, [60, 20], [2100, 30], 16, 1200), (8, 2, 128, [14, 1], [70, 900], 1024, 2400),
        (8, 2, 64, [1, 1, 2], [70, 900, 30], 1024, 4200)]


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("window,sinks", [(0, 0), (9, 2)])
@pytest.mark.parametrize("way", WAYS, ids=[f"{w[0]}x{w[2]}-{w[6]}" for w in WAYS])
def test_sums_that_are_not_finite_stay_with_what_the_query_sees(torch, way, window, sinks, value):   # noqa: F811
    heads, kv_heads, dim, new, lens, page, cols = way
    say(f"weights not finite {way} {window} {value}")
    b = Batch(torch, heads, kv_heads, dim, new, lens, page, cols=cols, seed=21)
    ref = b.reference(window=window, sinks=sinks, weights=b.weights)
    want, tol = ref[4], ref[5]
    i = max(range(len(new)), key=lambda r: new[r])
    t = (new[i] - 1) // 2   # later queries see tokens that it does not
    L, slot, head = lens[i], int(b.slots[i]), 1
    p = L - new[i] + t
    b.q[int(b.starts[i]) + t, head, 2] = value
    w = b.weights.clone()
    b.run(weights=w, window=window, sinks=sinks)
    assert b.kv.get_status() == OK
    j = torch.arange(w.shape[-1])
    seen = torch.zeros(w.shape, dtype=torch.bool)
    seen[slot, head // (heads // kv_heads)] = (j <= p) & ((j > p - window) | (j < sinks) if window else j >= 0)
    got = w.cpu()
    assert bool(torch.isnan(got[seen]).all())
    err = (got.double() - want).abs()
    assert bool((err <= tol)[~seen].all()), "tokens that it does not see"


def test_more_blocks_of_tokens_than_2_to_the_25(torch):   # noqa: F811
    """512 rows of 32,769 tokens (the same pages) and 1,024 KV heads, 69 GB of weights: every new token, which sees
    itself alone, has its 1."""
    from paper_2609_09800_amd import hbf
    rows, L, heads, dim, page, n = 512, 32769, 1024, 64, 16, 32
    say(f"weights of {rows} x {L} x {heads}")
    assert rows * -(-L // 512) * heads > 1 << 25
    i32 = dict(dtype=torch.int32, device="cuda")
    held = -(-L // page)
    pool = torch.zeros((1, 2, held, page, heads, dim), dtype=torch.bfloat16, device="cuda")
    kv = hbf.KvPages(pool, refs=torch.full((held,), rows, **i32), tables=torch.arange(held, **i32).repeat(rows, 1), lens=torch.full((rows,), L, **i32))
    q = torch.ones((rows * n, heads, dim), dtype=torch.bfloat16, device="cuda")
    out, w = torch.empty_like(q), torch.zeros((rows, heads, L), device="cuda")
    slots, starts = torch.arange(rows, **i32), torch.arange(0, rows * n + 1, n, **i32)
    assert kv.attention(0, q, out, slots, starts, weights=w, window=1) == OK and kv.get_status() == OK
    for at in range(0, rows, 64):
        new = w[at:at + 64, :, L - n:]
        assert bool((new == 1.0).all()), f"rows from {at}: {int((new != 1.0).sum())} without their weight"
        new.zero_()
        assert not bool(w[at:at + 64].any())
    del pool, kv, q, out, w, new
    torch.cuda.empty_cache()
