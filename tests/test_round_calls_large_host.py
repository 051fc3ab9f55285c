"""Sizes at the ends of what the attention call takes, on the host: its plan is made in whole numbers that hold them.  No GPU: nothing is launched."""
import ctypes as C

import pytest

import paper_2511_18191_amd as tsd
from paper_2511_18191_amd.binding import TsdPagedCache

L = tsd.lib()
PTR, OK, RANGE = 0x10000, 0, -3


def workspace(B, T, heads, max_len, kv_heads=16, head_dim=64, dtype=tsd.TSD_BF16):
    c = TsdPagedCache(PTR, PTR, 16 * kv_heads * head_dim, kv_heads * head_dim, head_dim, PTR, 8, 8, 100, 16, kv_heads, head_dim, dtype)
    n = C.c_size_t(12345)
    return L.tsd_paged_attn_workspace(C.byref(c), B, T, heads, max_len, C.byref(n)), n.value


@pytest.mark.parametrize("dtype", [tsd.TSD_BF16, tsd.TSD_F32])
@pytest.mark.parametrize("B,max_len", [(4096, 1 << 30), (65536, 1 << 26), (2048, 1 << 30), (1025, 1 << 30), (1 << 19, 1 << 30), (1024, (1 << 30) - 1)])
def test_many_sequences_of_any_length_stay_whole(dtype, B, max_len):
    # 16 key heads: more workgroups than are worth splitting, whatever max_len says
    assert workspace(B, 1, 16, max_len, dtype=dtype) == (OK, 0)


@pytest.mark.parametrize("T", [1, 17, 200])
@pytest.mark.parametrize("B", [1, 3, 16, 63])
@pytest.mark.parametrize("max_len", [(1 << 30) - 1, 1 << 30])
def test_parts_of_the_longest_caches(B, T, max_len):
    # split, into parts of 64 values and a logarithm a row; at most 16384 of them and one more a (key head, row tile), unless tall tiles are many
    rc, size = workspace(B, T, 4, max_len, kv_heads=4)
    row = B * T * 4 * (64 + 1) * 4
    tiles = B * 4 * (1 if T <= 64 else 2)
    splits = 16384 // tiles + 2
    assert rc == OK
    if T > 128 and tiles >= 256:
        assert size == 0
    else:
        assert 2 * row <= size <= splits * (row + 8 * tiles) + 256


@pytest.mark.parametrize("T", [(1 << 31) - 1, (1 << 31) - 40, (1 << 30) + 5])
@pytest.mark.parametrize("max_len", [1, 64, 1 << 30])
def test_as_many_rows_as_the_call_takes(T, max_len):
    rc, size = workspace(1, T, 1, max_len, kv_heads=1, head_dim=8)
    assert (rc, size) == (OK, 0)
