"""How attention cuts the prefix, from the scratch that a call asks for (the host's
part of it, without a GPU): the own tokens that a table's rows could hold must
not take the card from the prefix, as tables are as wide as a sequence may grow."""
import ctypes

import pytest

from paper_2609_09800_amd import hbf


def parts(rows, heads, kv_heads, dim, prefix, max_own):
    """Parts of the token axes, the prefix's and the own ones'."""
    lib = hbf.load_library()
    kv = hbf.hbf_kv_layer(None, None, 16 * kv_heads * dim, kv_heads * dim, dim, 1 << 20, 16, kv_heads, dim, hbf.HBF_BF16)
    at = hbf.hbf_attention(rows=rows, heads=heads, scale=1.0, prefix_len=prefix, max_own=max_own)
    b = ctypes.c_size_t()
    assert lib.hbf_kv_attention_workspace_bytes(ctypes.byref(kv), ctypes.byref(at), ctypes.byref(b)) == hbf.HBF_OK
    n, rest = divmod(b.value - 256, rows * heads * (dim * 4 + 8))
    assert rest == 0
    return n


@pytest.mark.parametrize("rows,heads,kv_heads,dim,prefix", [
    (64, 32, 4, 128, 32771), (64, 32, 4, 128, 4096), (16, 32, 4, 128, 4096), (1, 32, 4, 128, 4096), (8, 8, 8, 64, 9000)])
def test_the_prefix_keeps_its_parts_beside_a_wide_table(rows, heads, kv_heads, dim, prefix):
    alone = parts(rows, heads, kv_heads, dim, prefix, 0)
    narrow = parts(rows, heads, kv_heads, dim, prefix, 1024)
    for max_own in (2048, 8192, 32768, 131072, (1 << 31) - 1):
        assert parts(rows, heads, kv_heads, dim, prefix, max_own) >= max(narrow // 2, alone // 4)
