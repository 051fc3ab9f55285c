"""How much memory the calls with windows and trees ask for where batches are large and caches long.  No GPU: nothing is launched."""
import ctypes as C

import pytest

import paper_2511_18191_amd as tsd
from test_round_calls_host import L, cache

MOST = 256 << 20


def made(f, B, T, Hq, Hkv, D, max_len, window=0, sinks=0, dtype=tsd.TSD_BF16):
    n = C.c_size_t()
    c = cache(dtype=dtype, n_kv_heads=Hkv, head_dim=D, head_stride=D, token_stride=Hkv * D, page_stride=16 * Hkv * D)
    assert f(C.byref(c), B, T, Hq, max_len, window, sinks, C.byref(n)) == 0
    part = B * T * Hq * (D + 1) * 4                                            # a chunk's sums and logarithms
    return n.value // part, n.value % part, n.value


@pytest.mark.parametrize("dtype", [tsd.TSD_BF16, tsd.TSD_F32])
@pytest.mark.parametrize("Hq,Hkv,D", [(32, 8, 128), (16, 16, 64), (64, 16, 128), (32, 1, 80), (16, 4, 256), (128, 8, 128)])
def test_parts_are_bounded(dtype, Hq, Hkv, D):
    for B in (1, 2, 16, 64, 200, 1000):
        for T in (1, 8, 16, 33, 64, 256):
            for m in (100, 3000, 16384, 131072, 1 << 20, 1 << 30):
                for f, w, s in ((L.tsd_tree_attn_workspace, 0, 0), (L.tsd_tree_attn_workspace, 70000, 4), (L.tsd_window_attn_workspace, 70000, 4),
                                (L.tsd_window_attn_workspace, 1 << 30, 0)):
                    parts, rest, size = made(f, B, T, Hq, Hkv, D, m, w, s, dtype)
                    slots = 8 * B * Hkv * (T * Hq // Hkv // 16 + 1) * (MOST // (B * T * Hq * (D + 1) * 4) + 1)
                    assert size <= MOST + slots + 256, (B, T, m, parts)


def test_sequences_are_split_as_before_where_parts_are_small():
    # (chunks as they were measured: 16 x 64 nodes over up to 16384 keys, 32 over up to 8000, 4 and 1; 64 over up to 4096 whole)
    f = L.tsd_tree_attn_workspace
    for B, T, m, parts in ((16, 64, 16384, 6), (32, 64, 8000, 3), (4, 64, 16384, 8), (1, 64, 16384, 64), (64, 64, 4096, 0), (16, 64, 32768, 13)):
        assert made(f, B, T, 32, 8, 128, m)[0] == parts
