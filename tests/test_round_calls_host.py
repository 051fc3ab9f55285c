"""Host side of the calls for a round of the caller's own models: what they refuse before anything is launched, the plans and the
rotary frequencies.  No GPU: the pointers below are never followed."""
import ctypes as C
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from paper_2511_18191_amd.binding import TsdPagedCache, TsdRows

L = tsd.lib()
PTR, BAD, RANGE = 0x10000, -1, -3


def cache(**over):
    c = TsdPagedCache(PTR, PTR, 16 * 4 * 64, 4 * 64, 64, PTR, 8, 8, 100, 16, 4, 64, tsd.TSD_BF16)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def rows(**over):
    r = TsdRows(PTR, 4096, 512, 64)
    for k, v in over.items():
        setattr(r, k, v)
    return r


def said():
    return L.tsd_last_error(None).decode()


def append(c=None, B=2, T=3, H=8, q=None, out=None, k=None, v=None, base=PTR, freq=PTR, R=64, amplitude=1.0, flags=0):
    arg = lambda r: C.byref(r if r is not None else rows())
    return L.tsd_rope_append_static(C.byref(c or cache()), B, T, H, arg(q), arg(out), arg(k), arg(v), base, None, None, freq, R, amplitude, flags, None)


def attn(c=None, B=2, T=3, H=8, q=None, out=None, lens=PTR, max_len=128, scale=0.125, ws=None, nbytes=0):
    arg = lambda r: C.byref(r if r is not None else rows())
    return L.tsd_paged_attn_static(C.byref(c or cache()), B, T, H, arg(q), arg(out), None, lens, None, max_len, scale, ws, nbytes, None)


def verify(draft=PTR, p=PTR, dtype=tsd.TSD_F32, token_bytes=4, B=2, K=3, V=100, strides=(300, 100, 400, 100), u=PTR, n_acc=PTR, tokens=PTR, ws=PTR,
           nbytes=1 << 20):
    return L.tsd_verify_tokens_static(draft, None, p, dtype, token_bytes, B, K, V, *strides, u, None, n_acc, tokens, ws, nbytes, None)


@pytest.mark.parametrize("over,fragment", [
    (dict(k_dev=None), "NULL"), (dict(page_table_dev=None), "NULL"), (dict(dtype=2), "dtype"), (dict(page_tokens=12), "page_tokens"),
    (dict(page_tokens=2048), "page_tokens"), (dict(page_tokens=0), "page_tokens"), (dict(n_kv_heads=0), "n_kv_heads"), (dict(head_dim=60), "head_dim"),
    (dict(head_dim=264), "head_dim"), (dict(head_dim=0), "head_dim"), (dict(n_pages=0), "n_pages"), (dict(table_stride=7), "table_stride"),
    (dict(page_stride=-4096), "negative"), (dict(token_stride=4), "16 bytes"), (dict(k_dev=PTR + 8), "16 bytes"), (dict(head_stride=68), "16 bytes"),
])
def test_caches_that_are_refused(over, fragment):
    n = C.c_size_t()
    assert append(cache(**over)) == BAD and fragment in said()
    assert attn(cache(**over)) == BAD and fragment in said()
    assert L.tsd_paged_attn_workspace(C.byref(cache(**over)), 2, 3, 8, 128, C.byref(n)) == BAD


def test_cache_of_too_many_tokens():
    assert append(cache(pages_per_seq=1 << 28, table_stride=1 << 28)) == RANGE
    assert L.tsd_rope_append_static(None, 2, 3, 8, None, None, None, None, None, None, None, None, 64, 1.0, 0, None) == BAD and "cache" in said()


@pytest.mark.parametrize("over,fragment", [
    (dict(B=0), "B >= 1"), (dict(T=0), "T >= 1"), (dict(H=0), "n_q_heads"), (dict(H=1025), "n_q_heads"), (dict(q=rows(data_dev=None)), "q must"),
    (dict(q=rows(stride_t=12)), "q:"), (dict(out=rows(data_dev=PTR + 2)), "q_out"), (dict(k=rows(stride_h=-8)), "k:"), (dict(v=rows(stride_b=4)), "v:"),
    (dict(base=None), "base_dev"), (dict(freq=None), "freq_dev"), (dict(R=63), "rotary_dim"), (dict(R=66), "rotary_dim"), (dict(R=0), "rotary_dim"),
    (dict(amplitude=math.inf), "amplitude"), (dict(flags=tsd.TSD_FLAG_NO_GRAPH), "flags"),
])
def test_appends_that_are_refused(over, fragment):
    assert append(**over) == BAD and fragment in said()
    assert append(B=1 << 16, T=1 << 16) == RANGE


@pytest.mark.parametrize("over,fragment", [
    (dict(B=0), "B >= 1"), (dict(T=0), "T >= 1"), (dict(H=6), "multiple"), (dict(H=0), "multiple"), (dict(max_len=0), "max_len"),
    (dict(max_len=(1 << 30) + 1), "max_len"), (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"), (dict(lens=None), "lens_dev"),
    (dict(q=rows(stride_b=3)), "q:"), (dict(out=rows(data_dev=None)), "out"), (dict(max_len=20000), "workspace"),
    (dict(max_len=20000, ws=PTR, nbytes=64), "workspace"), (dict(max_len=20000, ws=PTR + 4, nbytes=1 << 30), "workspace"),
])
def test_attentions_that_are_refused(over, fragment):
    assert attn(**over) == BAD and fragment in said()
    assert attn(B=1 << 20, T=1 << 10) == RANGE


@pytest.mark.parametrize("over,fragment", [
    (dict(draft=None), "NULL"), (dict(p=None), "NULL"), (dict(u=None), "NULL"), (dict(n_acc=None), "NULL"), (dict(tokens=None), "NULL"),
    (dict(dtype=7), "dtype"), (dict(token_bytes=2), "token_bytes"), (dict(B=0), "B >= 1"), (dict(K=0), "K >= 1"), (dict(V=0), "V >= 1"),
    (dict(strides=(-1, 1, 1, 1)), "strides"), (dict(strides=(1, 1, 1, -1)), "strides"), (dict(ws=None), "workspace"), (dict(nbytes=0), "workspace"),
    (dict(ws=PTR + 4), "workspace"),
])
def test_verifications_that_are_refused(over, fragment):
    assert verify(**over) == BAD and fragment in said()
    assert verify(K=17) == RANGE and verify(B=1 << 30, V=1 << 20) == RANGE


def test_workspaces():
    n = C.c_size_t()
    need = lambda B, T, H, m, c=None: (L.tsd_paged_attn_workspace(C.byref(c or cache()), B, T, H, m, C.byref(n)), n.value)
    assert need(1, 1, 4, 100) == (0, 0)                       # short caches, and many sequences, are not split
    assert need(4096, 1, 4, 1 << 14) == (0, 0)
    for T, m in ((1, 5000), (5, 32768), (17, 1 << 20)):       # parts of 64 values and a logarithm each, at most some 1000 per key head
        rc, size = need(1, T, 4, m)
        row = T * 4 * (64 + 1) * 4
        assert rc == 0 and 2 * row <= size <= 2048 * row + 256
    assert L.tsd_paged_attn_workspace(C.byref(cache()), 1, 1, 4, 100, None) == BAD
    assert L.tsd_verify_tokens_workspace(3, 4, 32000, tsd.TSD_BF16, C.byref(n)) == 0 and n.value >= 3 * 8
    assert L.tsd_verify_tokens_workspace(3, 4, 32000, tsd.TSD_BF16, None) == BAD


def test_rotary_frequencies():
    R, base, s = 64, 10000.0, 4.0
    plain, amp = tsd.rope_frequencies(R, base, device="cpu")
    assert plain.dtype == torch.float64 and amp == 1.0
    assert plain.tolist() == pytest.approx([base ** (-2 * i / R) for i in range(R // 2)], rel=1e-14)
    linear, amp = tsd.rope_frequencies(R, base, "linear", s, device="cpu")
    assert torch.allclose(linear * s, plain, rtol=1e-14, atol=0) and amp == 1.0
    stretched, _ = tsd.rope_frequencies(R, base, "base", s, device="cpu")
    assert float(stretched[0]) == 1.0 and float(stretched[-1] * s) == pytest.approx(float(plain[-1]), rel=1e-12)
    blend, amp = tsd.rope_frequencies(R, base, "blend", s, original_len=4096, low=1.0, high=32.0, device="cpu")
    turns = 4096 * plain / (2 * math.pi)
    fast, slow = turns >= 32, turns <= 1
    assert fast.any() and slow.any() and not (fast | slow).all()
    assert torch.equal(blend[fast], plain[fast]) and torch.allclose(blend[slow] * s, plain[slow], rtol=1e-14, atol=0)
    keep = ((turns - 1) / 31)[~(fast | slow)]
    assert torch.allclose(blend[~(fast | slow)], plain[~(fast | slow)] * (keep + (1 - keep) / s), rtol=1e-13, atol=0)
    assert amp == pytest.approx(0.1 * math.log(s) + 1)
    with pytest.raises(ValueError):
        tsd.rope_frequencies(R, scaling="other", device="cpu")
    for bad in (dict(rotary_dim=63), dict(rotary_dim=0), dict(rotary_dim=258), dict(rotary_dim=64, base=1.0), dict(rotary_dim=64, base=math.nan),
                dict(rotary_dim=64, scaling="linear", factor=0.5), dict(rotary_dim=2, scaling="base", factor=2.0),
                dict(rotary_dim=64, scaling="blend", factor=2.0), dict(rotary_dim=64, scaling="blend", factor=2.0, original_len=9, low=3.0, high=2.0)):
        with pytest.raises(tsd.TsdError):
            tsd.rope_frequencies(device="cpu", **bad)


def test_tensors_of_the_host_and_what_is_no_tensor():
    z = torch.zeros
    q, kv, pool, table, base = z(2, 3, 4, 64), z(2, 3, 4, 64), z(9, 16, 4, 64), z(2, 4, dtype=torch.int32), z(2, dtype=torch.int32)
    freq, p, draft = z(32, dtype=torch.float64), z(2, 4, 10), z(2, 3, dtype=torch.int64)
    for call in (lambda: tsd.rope_append_static(q, kv, kv, pool, pool, table, base, freq), lambda: tsd.paged_attn_static(q, pool, pool, table, base),
                 lambda: tsd.verify_tokens_static(draft, p[:, :3], p, z(2, 4))):
        with pytest.raises(ValueError, match="cuda"):
            call()
    for call in (lambda: tsd.rope_append_static(q, kv, None, pool, pool, table, base, freq), lambda: tsd.paged_attn_static(q, pool, pool, [[0]], base),
                 lambda: tsd.verify_tokens_static(draft.tolist(), None, p, z(2, 4))):
        with pytest.raises(TypeError, match="tensor"):
            call()
    with pytest.raises(ValueError, match="max_len"):
        tsd.paged_attn_static(q, pool, pool, table, base, max_len=0)
    with pytest.raises(ValueError, match="scale"):
        tsd.paged_attn_static(q, pool, pool, table, base, scale=math.nan)
