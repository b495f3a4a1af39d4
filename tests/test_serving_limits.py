"""Serving from a cache of pages, calls at and past the largest sizes, on the host (no GPU)."""
import ctypes

import pytest

from paper_2609_09800_amd import hbf
from test_scratch_streams import Block, notes  # noqa: F401
from test_serving_host import AT, EINVAL, OK, cache, call_chunk, chunk, layer, lib, objects  # noqa: F401


@pytest.mark.parametrize("rows,kv_heads,tokens,heads,rc", [
    (65535, 257, 1, 257, EINVAL), (65535, 1024, 1, 1024, EINVAL), (65535, 256, 16, 256, EINVAL), (62000, 256, 1 << 15, 512, EINVAL),
    (65535, 256, 14, 256, OK), (61439, 256, 1 << 15, 512, OK), (65535, 1, 1 << 20, 16, OK), (15000, 1024, 1, 1024, OK)])
def test_attention_refuses_more_workgroups_than_a_launch_takes(lib, rows, kv_heads, tokens, heads, rc):   # noqa: F811
    """A tile of 16 queries and a KV head a workgroup of 256 threads: one launch has fewer than 2^32 threads."""
    b, c, l = ctypes.c_size_t(), cache(), layer(kv_heads=kv_heads)
    for weights in (None, AT):
        h = chunk(rows=rows, tokens=tokens, heads=heads, dev_weights=weights, weights_tokens=64)
        assert lib.hbf_kv_chunk_workspace_bytes(ctypes.byref(c), ctypes.byref(l), ctypes.byref(h), ctypes.byref(b)) == rc
        if rc != OK:
            assert call_chunk(lib, c, l, h) == rc
        else:   # every workgroup that such a call starts
            assert (rows + (tokens * (heads // kv_heads) >> 4)) * kv_heads * 256 < 1 << 32


@pytest.mark.parametrize("how", [dict(window=2 ** 31), dict(window=2 ** 32 + 5), dict(sinks=2 ** 31), dict(sinks=-2 ** 31 - 1), dict(window=10 ** 30)])
def test_attention_refuses_numbers_that_do_not_fit(notes, how):   # noqa: F811
    kv = objects(notes)
    q, out, slots, starts = (Block(notes, s, d) for s, d in (((9, 4, 64), "bf16"), ((9, 4, 64), "bf16"), ((3,), "int32"), ((4,), "int32")))
    with pytest.raises(hbf.HbfError, match=f"{next(iter(how))}.*fit"):
        kv.attention(0, q, out, slots, starts, **how)
    assert not notes.calls
    for ok in (dict(window=2 ** 31 - 1, sinks=2 ** 31 - 1), dict(window=-2 ** 31), dict(scale=1e39)):   # (the library looks at these)
        assert kv.attention(0, q, out, slots, starts, **ok) == OK


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32 + 3])
def test_write_rotated_refuses_numbers_that_do_not_fit(notes, monkeypatch, n):   # noqa: F811
    monkeypatch.setattr(hbf.torch, "float64", "float64", raising=False)
    kv = objects(notes)
    k, v, slots, pos, freqs = (Block(notes, s, d) for s, d in (((n, 1, 64), "bf16"), ((n, 1, 64), "bf16"), ((n,), "int32"), ((n,), "int32"), ((32,), "float64")))
    q, out = Block(notes, (n, 4, 64), "bf16"), Block(notes, (n, 4, 64), "bf16")
    with pytest.raises(hbf.HbfError, match="tokens.*fit"):
        kv.write_rotated(0, q, k, v, slots, pos, freqs, out)
    assert not notes.calls


@pytest.mark.parametrize("what,value", [("sinks", 2 ** 32), ("recent", 2 ** 32 + 8), ("recent", 2 ** 31), ("sinks", -2 ** 32),
                                        ("max_keep", 2 ** 32)])
def test_evict_refuses_numbers_that_do_not_fit(notes, what, value):   # noqa: F811
    """(Cut to 32 bits they would be other numbers, 0 and 8 among them.)"""
    kv = objects(notes)
    slots, keep, w, kept = (Block(notes, s, d) for s, d in (((3,), "int32"), ((3,), "int32"), ((2, 8, 1, 64), "float32"), ((2, 3, 1, value if what == "max_keep" else 40), "int32")))
    with pytest.raises(hbf.HbfError, match=f"{what}.*fit"):
        kv.evict(slots, keep, w, kept, **({} if what == "max_keep" else {what: value}))
    assert not notes.calls
