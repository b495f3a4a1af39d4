"""Which tiles attention over pages takes, from the scratch that a call asks for (the
host's part of it, without a GPU): the GPU tests' cases reach the tiles that they
are there for."""
import ctypes

import pytest

from paper_2609_09800_amd import hbf
from test_gpu_chunk_attention import CASES, SHAPES, WIDE_CASES
from test_serving_host import AT, OK, cache, chunk, layer


def scratch(heads, kv_heads, dim, new, lens, page, cols, tokens):
    held = max(-(-max(lens) // page), 0) + 1 + cols
    kv = cache(page_tokens=page, table_cols=held, table_stride=held, slots=len(lens) + 1, token_bytes=2 * kv_heads * dim,
               page_stride=2 * kv_heads * dim * page)
    ly = layer(page_tokens=page, kv_heads=kv_heads, head_dim=dim)
    ch = chunk(tokens=tokens, rows=len(new), heads=heads, dev_ctl=AT)
    b = ctypes.c_size_t()
    assert hbf.load_library().hbf_kv_chunk_workspace_bytes(ctypes.byref(kv), ctypes.byref(ly), ctypes.byref(ch), ctypes.byref(b)) == OK
    return b.value


def tiles(need, heads, kv_heads, dim, new, tokens):
    """The tiles, 16 or 256 queries, whose parts take as much: sums and maxima of every tile, KV head and part, a
    workgroup each, which are all on the card at once (four a CU at the most)."""
    up = lambda n: -(-n // 256) * 256
    fits = set()
    for q in (16, 256):
        slots = tokens * (heads // kv_heads) // q + len(new)
        for parts in range(2, 1024 // (slots * kv_heads) + 1):
            n = slots * kv_heads * parts * q
            if need == up(n * dim * 4) + up(n * 8):
                fits.add(q)
    return fits


@pytest.mark.parametrize("case", WIDE_CASES, ids=str)
def test_wide_cases_are_cut_into_tiles_of_256(case):
    heads, kv_heads, dim, new, lens, page = case[:6]
    tokens = sum(new) + 3   # (some lie before and behind the rows)
    assert tiles(scratch(heads, kv_heads, dim, new, lens, page, 19200 // page, tokens), heads, kv_heads, dim, new, tokens) == {256}


@pytest.mark.parametrize("case", CASES, ids=str)
def test_other_cases_are_cut_into_tiles_of_16(case):
    heads, kv_heads, dim, new, lens, page = case[:6]
    tokens = sum(new) + 3
    need = scratch(heads, kv_heads, dim, new, lens, page, 0, tokens)
    assert need == 256 or tiles(need, heads, kv_heads, dim, new, tokens) == {16}   # (256: not in parts)


@pytest.mark.parametrize("shape,tile", list(zip(SHAPES, (16, 16, 256, 256))), ids=str)
def test_shapes(shape, tile):
    heads, kv_heads, dim, new, lens, page, cols = shape
    need = scratch(heads, kv_heads, dim, new, lens, page, cols, sum(new))
    assert tile == 16 and need == 256 or tiles(need, heads, kv_heads, dim, new, sum(new)) == {tile}
