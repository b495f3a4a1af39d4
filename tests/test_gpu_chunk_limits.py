"""Attention over pages with as many workgroups as one launch takes."""
import pytest

from test_gpu_chunk_attention import EINVAL, OK, U, say, torch  # noqa: F401

pytestmark = pytest.mark.gpu


def test_as_many_rows_and_heads_as_a_launch_takes(torch):   # noqa: F811
    """65,535 rows of 256 KV heads, 14 of them with a token, which sees itself alone: its result is its V."""
    from paper_2609_09800_amd import hbf
    rows, heads, dim, tokens = 65535, 256, 64, 14
    say(f"attention {rows} rows of {heads} heads")
    gen = torch.Generator(device="cuda").manual_seed(41)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.randn((1, 2, tokens, 1, heads, dim), generator=gen, device="cuda").bfloat16()
    lens = torch.ones(tokens + 1, **i32)
    lens[tokens] = 0
    kv = hbf.KvPages(pool, refs=torch.ones(tokens, **i32), tables=torch.arange(tokens + 1, **i32).view(-1, 1).clamp(max=tokens - 1), lens=lens)
    at = torch.linspace(0, rows - 1, tokens, device="cuda").long()   # the rows that have a token
    slots, new = torch.full((rows,), tokens, **i32), torch.zeros(rows, **i32)
    slots[at], new[at] = torch.arange(tokens, **i32), 1
    starts = torch.cat([torch.zeros(1, **i32), torch.cumsum(new, 0, dtype=torch.int32)])
    q = torch.randn((tokens + 1, heads, dim), generator=gen, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    n = tokens
    assert kv.attention(0, q[:n], out[:n], slots, starts, lse=lse[:n]) == OK and kv.get_status() == OK
    v = pool[0, 1, :, 0].float()
    k = pool[0, 0, :, 0].double()
    ds = (dim + 8) * 2.0 ** -23 * float((q[:n].double().abs() * k.abs()).sum(-1).max()) / 8
    assert bool(((out[:n].float() - v).abs() <= (2 * U["bfloat16"] + 2 * ds + 17 * 2.0 ** -23) * v.abs()).all())
    want = (q[:n].double() * k).sum(-1) / 8
    assert bool(((lse[:n].double() - want).abs() <= ds + 17 * 2.0 ** -23 + 2.0 ** -22 * want.abs()).all())
    # a workgroup's worth more is refused
    q, out = q.repeat(2, 1, 1)[:16], out.repeat(2, 1, 1)[:16]
    assert kv.attention(0, q, out, slots, starts) == EINVAL
