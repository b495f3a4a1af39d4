"""Serving from a cache of pages, the host's part (no GPU): what the C entries
refuse before any launch, the waits before a hand-over (read from the source), and
the blocks and streams of the objects."""
import ctypes
import re

import pytest

from paper_2609_09800_amd import hbf
from test_hand_over_waits import source
from test_scratch_streams import Block, known, notes  # noqa: F401

EINVAL, OK, ENOWS = hbf.HBF_EINVAL, hbf.HBF_OK, hbf.HBF_ENOWORKSPACE
AT = 1 << 20   # an address that is aligned; nothing behind it is looked at


@pytest.fixture(scope="module")
def lib():
    return hbf.load_library()


def cache(**kw):
    d = dict(dev_pool=AT, plane_stride=64 * 16 * 256, page_stride=16 * 256, token_bytes=256, planes=4, pages=64,
             page_tokens=16, slots=8, table_cols=32, table_stride=32, dev_refs=AT, dev_tables=AT, dev_lens=AT, dev_ws=AT)
    return hbf.hbf_kv(**{**d, **kw})


def layer(**kw):
    d = dict(dev_k=AT, dev_v=AT, page_stride=16 * 128, token_stride=128, head_stride=64, pages=64, page_tokens=16,
             kv_heads=2, head_dim=64, dtype=hbf.HBF_BF16)
    return hbf.hbf_kv_layer(**{**d, **kw})


def chunk(**kw):
    d = dict(dev_q=AT, q_row_stride=512, q_head_stride=64, tokens=20, rows=3, heads=8, scale=0.125, dev_slots=AT,
             dev_starts=AT, dev_out=AT, out_row_stride=512, out_head_stride=64)
    return hbf.hbf_chunk(**{**d, **kw})


def call_chunk(lib, kv=None, ly=None, ch=None, ws=AT, nbytes=1 << 40, status=0):
    ref = lambda x: ctypes.byref(x) if x is not None else None
    return lib.hbf_kv_chunk_attention(ref(kv), ref(ly), ref(ch), status, ws, nbytes, None)


def test_attention_refuses(lib):
    no = [
        (dict(kv=None), {}), (dict(ly=None), {}), (dict(ch=None), {}),
        *((dict(kv=cache(**k)), {}) for k in (dict(slots=0), dict(pages=0), dict(page_tokens=8), dict(table_stride=31),
                                              dict(dev_tables=None), dict(dev_lens=None), dict(dev_tables=AT + 2))),
        *((dict(ly=layer(**k)), {}) for k in (dict(head_dim=96), dict(kv_heads=0), dict(kv_heads=3), dict(dtype=7),
                                              dict(dev_k=None), dict(dev_v=AT + 8), dict(token_stride=12), dict(pages=0))),
        *((dict(ch=chunk(**k)), {}) for k in (
            dict(tokens=-1), dict(tokens=(1 << 20) + 1), dict(tokens=1 << 20, heads=32), dict(rows=-1), dict(rows=65536),
            dict(heads=7), dict(heads=0), dict(heads=1026), dict(scale=float("inf")), dict(scale=float("nan")),
            dict(window=-1), dict(sinks=-1), dict(q_row_stride=4), dict(out_head_stride=60), dict(dev_q=None),
            dict(dev_q=AT + 8), dict(dev_out=None), dict(dev_out=AT + 2), dict(dev_lse=AT + 2), dict(dev_slots=None),
            dict(dev_starts=None), dict(dev_starts=AT + 1), dict(dev_weights=AT + 2), dict(weights_tokens=-1),
            dict(weights_slot_stride=-1), dict(weights_head_stride=-1), dict(dev_ctl=AT + 2))),
        ({}, dict(ws=None)), ({}, dict(ws=AT + 64)), ({}, dict(status=AT + 1)),
    ]
    for parts, how in no:
        args = {**dict(kv=cache(), ly=layer(), ch=chunk()), **parts}
        assert call_chunk(lib, **args, **how) == EINVAL, (parts, how)
    assert call_chunk(lib, cache(), layer(), chunk(rows=0)) == OK      # nothing to do
    assert call_chunk(lib, cache(), layer(), chunk(tokens=0)) == OK
    b = ctypes.c_size_t()
    c, l, h = cache(), layer(), chunk()
    assert lib.hbf_kv_chunk_workspace_bytes(ctypes.byref(c), ctypes.byref(l), ctypes.byref(h), ctypes.byref(b)) == OK
    assert b.value > 0 and call_chunk(lib, c, l, h, nbytes=b.value - 1) == ENOWS
    assert lib.hbf_kv_chunk_workspace_bytes(ctypes.byref(c), ctypes.byref(l), ctypes.byref(h), None) == EINVAL


@pytest.mark.parametrize("rows,tokens,heads", [(0, 0, 8), (0, 1, 2), (0, 20, 8), (3, 0, 8), (1, 1, 2)])
def test_scratch_of_calls_with_little_or_nothing_to_do(lib, rows, tokens, heads):
    for more in (dict(), dict(dev_ctl=AT), dict(dev_ctl=AT, dev_weights=AT, weights_tokens=0),
                 dict(dev_weights=AT, weights_tokens=2 ** 31 - 1)):
        b, c, l, h = ctypes.c_size_t(), cache(), layer(), chunk(rows=rows, tokens=tokens, heads=heads, **more)
        assert lib.hbf_kv_chunk_workspace_bytes(ctypes.byref(c), ctypes.byref(l), ctypes.byref(h), ctypes.byref(b)) == OK
        assert b.value >= 256
        if not rows or not tokens:
            assert call_chunk(lib, c, l, h) == OK


def test_write_rotated_refuses(lib):
    def call(kv={}, at=0, **kw):
        d = dict(dev_q=AT, dev_k=AT, dev_v=AT, q_row_stride=512, q_head_stride=64, k_row_stride=128, k_head_stride=64,
                 v_row_stride=128, v_head_stride=64, dev_q_out=AT, out_row_stride=512, out_head_stride=64, n=5, heads=8,
                 kv_heads=2, head_dim=64, dtype=hbf.HBF_BF16, eps=1e-6, pairs=32, dev_freqs=AT, dev_slots=AT, dev_pos=AT)
        return lib.hbf_kv_write_rotated(ctypes.byref(cache(**kv)), at, ctypes.byref(hbf.hbf_new_tokens(**{**d, **kw})), None)

    assert call(n=0) == OK
    assert lib.hbf_kv_write_rotated(ctypes.byref(cache()), 0, None, None) == EINVAL
    assert lib.hbf_kv_write_rotated(None, 0, ctypes.byref(hbf.hbf_new_tokens()), None) == EINVAL
    for kw in (dict(n=-1), dict(n=(1 << 20) + 1), dict(heads=0), dict(heads=1025), dict(kv_heads=0), dict(kv_heads=1),
               dict(head_dim=128), dict(head_dim=32), dict(dtype=3), dict(flags=2), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(pairs=-8), dict(pairs=4), dict(pairs=40), dict(dev_freqs=None), dict(dev_freqs=AT + 4),
               dict(dev_q=None), dict(dev_k=AT + 8), dict(dev_v=None), dict(dev_q_out=AT + 2), dict(dev_slots=None),
               dict(dev_pos=AT + 1), dict(dev_positions=AT + 2), dict(dev_q_weight=AT + 8), dict(dev_k_weight=AT + 8),
               dict(q_row_stride=4), dict(v_head_stride=3), dict(out_row_stride=1), dict(at=2), dict(at=-1),
               dict(kv=dict(dev_ws=None)), dict(kv=dict(dev_pool=AT + 8)), dict(kv=dict(token_bytes=128))):
        assert call(**kw) == EINVAL, kw


def test_evict_refuses(lib):
    def call(kv={}, **kw):
        d = dict(dev_slots=AT, dev_keep=AT, n=2, kv_heads=2, sinks=4, recent=8, dev_weights=AT, layer_stride=8192,
                 slot_stride=1024, head_stride=512, weights_tokens=512, dev_kept=AT, max_keep=100)
        return lib.hbf_kv_evict(ctypes.byref(cache(**kv)), ctypes.byref(hbf.hbf_eviction(**{**d, **kw})), None)

    assert call(n=0) == OK
    assert lib.hbf_kv_evict(ctypes.byref(cache()), None, None) == EINVAL
    for kw in (dict(n=-1), dict(n=65536), dict(kv_heads=0), dict(kv_heads=32), dict(kv_heads=1025), dict(sinks=-1),
               dict(recent=-1), dict(weights_tokens=-1), dict(max_keep=-1), dict(max_keep=(1 << 24) + 1), dict(layer_stride=-1),
               dict(slot_stride=-1), dict(head_stride=-1), dict(dev_slots=None), dict(dev_keep=None), dict(dev_weights=None),
               dict(dev_kept=None), dict(dev_kept=AT + 2), dict(dev_weights=AT + 1), dict(dev_weights_out=AT + 3),
               dict(kv=dict(planes=3)), dict(kv=dict(dev_ws=AT + 16)),
               dict(n=65535, kv_heads=16, kv=dict(planes=20))):   # more choices than a launch takes
        assert call(**kw) == EINVAL, kw


@pytest.mark.parametrize("file", ["hbf_chunk.hip", "hbf_evict.hip"])
def test_every_last_of_comes_right_after_a_wait(file):
    calls = list(re.finditer(r"if \(!?last_of\(", source(file)))
    assert calls
    for m in calls:
        assert source(file)[:m.start()].rstrip().endswith("stores_done();")


def objects(notes):   # noqa: F811
    pool = Block(notes, (2, 2, 64, 16, 1, 64), "bf16")
    return hbf.KvPages(pool, refs=Block(notes, (64,)), tables=Block(notes, (8, 4)), lens=Block(notes, (8,)))


def test_blocks_are_known_on_every_stream(notes, monkeypatch):   # noqa: F811
    monkeypatch.setattr(hbf.torch, "float64", "float64", raising=False)
    kv = objects(notes)
    q, out, slots, starts = (Block(notes, s, d) for s, d in (((9, 4, 64), "bf16"), ((9, 4, 64), "bf16"), ((3,), "int32"), ((4,), "int32")))
    known(notes, lambda: [kv._attn_status, kv._attn_ws._t], lambda stream: kv.attention(0, q, out, slots, starts, stream=stream))
    notes.current = type(notes.current)(1)
    kv = objects(notes)
    k, v, pos, freqs = (Block(notes, s, d) for s, d in (((3, 1, 64), "bf16"), ((3, 1, 64), "bf16"), ((3,), "int32"), ((32,), "float64")))
    q, out = Block(notes, (3, 4, 64), "bf16"), Block(notes, (3, 4, 64), "bf16")
    known(notes, lambda: [kv._ws], lambda stream: kv.write_rotated(0, q, k, v, slots, pos, freqs, out, stream=stream))
    notes.current = type(notes.current)(1)
    kv = objects(notes)
    w, kept = Block(notes, (2, 8, 1, 64), "float32"), Block(notes, (2, 3, 1, 40))
    known(notes, lambda: [kv._ws], lambda stream: kv.evict(slots, pos, w, kept, stream=stream))
