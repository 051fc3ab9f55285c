"""Into how many parts the attention call splits the keys of prompts, by the workspace it asks for.  No GPU: nothing is launched."""
import ctypes as C

import pytest

import paper_2511_18191_amd as tsd
from paper_2511_18191_amd.binding import TsdPagedCache

L = tsd.lib()


def parts(B, T, heads, kv_heads, D, max_len):
    c = TsdPagedCache(0x10000, 0x10000, 16 * kv_heads * D, kv_heads * D, D, 0x10000, 64, 64, 100, 16, kv_heads, D, tsd.TSD_BF16)
    n = C.c_size_t()
    assert L.tsd_paged_attn_workspace(C.byref(c), B, T, heads, max_len, C.byref(n)) == 0
    return n.value // (B * T * heads * (D + 1) * 4) if n.value else 1


@pytest.mark.parametrize("B,T,heads,kv_heads,D", [(1, 17, 8, 2, 128), (1, 75, 4, 4, 80), (3, 128, 2, 2, 32)])
def test_short_prompts(B, T, heads, kv_heads, D):
    # whole up to 256 keys, then at most eight parts until these are of 256 keys
    assert [parts(B, T, heads, kv_heads, D, n) for n in (1, 64, 200, 256)] == [1] * 4
    assert [parts(B, T, heads, kv_heads, D, n) for n in (257, 512, 513, 1024, 1025, 2048)] == [5, 8, 5, 8, 6, 8]
    assert parts(B, T, heads, kv_heads, D, 4096) == 16
