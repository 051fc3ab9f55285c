"""Host side of the calls for rounds of trees, windowed caches and scores: what they refuse before anything is launched, and their workspaces.  No GPU: the
pointers below are never followed."""
import ctypes as C
import math
import sys
import types

import pytest
import torch

import paper_2511_18191_amd as tsd
from paper_2511_18191_amd import binding
from test_round_calls_host import BAD, L, PTR, RANGE, cache, rows, said


def window(c=None, B=2, T=3, H=8, q=None, out=None, lens=PTR, max_len=128, window=50, sinks=4, scale=0.125, ws=None, nbytes=0):
    arg = lambda r: C.byref(r if r is not None else rows())
    return L.tsd_window_attn_static(C.byref(c or cache()), B, T, H, arg(q), arg(out), None, lens, None, max_len, window, sinks, scale, ws, nbytes, None)


def tree(c=None, B=2, T=3, H=8, q=None, out=None, lens=PTR, max_len=128, window=0, sinks=0, scale=0.125, parents=PTR, stride=0, ws=None, nbytes=0):
    arg = lambda r: C.byref(r if r is not None else rows())
    return L.tsd_tree_attn_static(C.byref(c or cache()), B, T, H, arg(q), arg(out), None, lens, None, parents, stride, max_len, window, sinks, scale, ws, nbytes,
                                  None)


def scores(logits=PTR, dtype=tsd.TSD_F32, token_bytes=8, B=2, T=3, V=100, strides=(300, 100), tokens=PTR, temperature=1.0, top=4, lp=PTR, ent=PTR, ids=PTR,
           alt=PTR, ws=PTR, nbytes=1 << 20):
    return L.tsd_token_logprobs_static(logits, dtype, token_bytes, B, T, V, *strides, tokens, None, temperature, top, lp, ent, ids, alt, ws, nbytes, None)


def walk(tokens=PTR, parents=PTR, stride=0, p=PTR, dtype=tsd.TSD_F32, token_bytes=4, B=2, N=5, V=100, strides=(500, 100), u=PTR, choices=None, n_acc=PTR,
         out=PTR, path=PTR, ws=PTR, nbytes=1 << 30):
    return L.tsd_verify_tree_static(tokens, parents, stride, p, dtype, token_bytes, B, N, V, *strides, u, choices, None, n_acc, out, path, ws, nbytes, None)


def keep(c=None, layers=1, stride=0, B=2, N=5, held=PTR, path=PTR):
    return L.tsd_keep_path_static(C.byref(c or cache()), layers, stride, B, N, held, path, None)


@pytest.mark.parametrize("over,fragment", [
    (dict(k_dev=None), "NULL"), (dict(page_table_dev=None), "NULL"), (dict(dtype=2), "dtype"), (dict(page_tokens=12), "page_tokens"), (dict(head_dim=60), "head_dim"),
    (dict(n_pages=0), "n_pages"), (dict(table_stride=7), "table_stride"), (dict(page_stride=-4096), "negative"), (dict(k_dev=PTR + 8), "16 bytes"),
])
def test_caches_that_are_refused(over, fragment):
    for call in (window, tree, keep):
        assert call(cache(**over)) == BAD and fragment in said()


@pytest.mark.parametrize("over,fragment", [
    (dict(B=0), "B >= 1"), (dict(T=0), "T >= 1"), (dict(H=6), "multiple"), (dict(max_len=0), "max_len"), (dict(max_len=(1 << 30) + 1), "max_len"),
    (dict(scale=math.nan), "scale"), (dict(lens=None), "lens_dev"), (dict(q=rows(stride_b=3)), "q:"), (dict(out=rows(data_dev=None)), "out"),
    (dict(window=-1), "window"), (dict(sinks=-1), "sinks"), (dict(max_len=20000, window=20000), "workspace"),
    (dict(max_len=20000, window=20000, ws=PTR + 4, nbytes=1 << 30), "workspace"),
])
def test_attentions_that_are_refused(over, fragment):
    for call in (window, tree):
        assert call(**over) == BAD and fragment in said()
        assert call(B=1 << 20, T=1 << 8, H=16) == RANGE
    assert window(window=0) == BAD and "window" in said()
    assert tree(T=257) == RANGE and "256" in said()
    assert tree(parents=None) == BAD and "parents" in said()
    assert tree(stride=2) == BAD and tree(stride=-3) == BAD and "parents_stride" in said()


@pytest.mark.parametrize("over,fragment", [
    (dict(logits=None), "NULL"), (dict(ent=None), "NULL"), (dict(tokens=None), "together"), (dict(lp=None), "together"), (dict(ids=None), "beside top"),
    (dict(alt=None), "beside top"), (dict(dtype=7), "dtype"), (dict(token_bytes=2), "token_bytes"), (dict(B=0), "B >= 1"), (dict(T=0), "T >= 1"), (dict(V=0), "V >= 1"),
    (dict(strides=(-1, 1)), "strides"), (dict(strides=(1, -1)), "strides"), (dict(temperature=0.0), "temperature"), (dict(temperature=-1.0), "temperature"),
    (dict(temperature=math.nan), "temperature"), (dict(temperature=math.inf), "temperature"), (dict(temperature=1e-7), "temperature"), (dict(top=-1), "top"),
    (dict(V=100000, ws=None), "workspace"), (dict(V=100000, nbytes=8), "workspace"), (dict(V=100000, ws=PTR + 4), "workspace"),
])
def test_scores_that_are_refused(over, fragment):
    assert scores(**over) == BAD and fragment in said()
    assert scores(top=33) == RANGE and scores(V=(1 << 23) + 1) == RANGE and scores(B=1 << 15, T=1 << 15) == RANGE


def test_scores_of_as_many_rows_as_a_launch_takes():
    n = C.c_size_t(1)
    most = 0xFFFFFFFF // 256  # workgroups of 256 lanes: one a row of up to 262144 logits
    for B, T, V, rc in ((most, 1, 32000, 0), (1024, 4096, 32000, 0), (most + 1, 1, 32000, RANGE), (1 << 30, 1 << 30, 8, RANGE), (most // 2, 1, 262145, 0),
                        (most // 2 + 1, 1, 262145, RANGE)):
        assert L.tsd_token_logprobs_workspace(B, T, V, 5, C.byref(n)) == rc
        assert rc or (n.value == 0) == (V <= 262144)


@pytest.mark.parametrize("over,fragment", [
    (dict(tokens=None), "NULL"), (dict(parents=None), "NULL"), (dict(n_acc=None), "NULL"), (dict(out=None), "NULL"), (dict(path=None), "NULL"), (dict(p=None), "either"),
    (dict(choices=PTR), "either"), (dict(u=None), "uniforms"), (dict(dtype=5), "dtype"), (dict(token_bytes=1), "token_bytes"), (dict(stride=4), "parents_stride"),
    (dict(stride=-5), "parents_stride"), (dict(strides=(-1, 1)), "strides"), (dict(B=0), "B >= 1"), (dict(N=0), "N >= 1"), (dict(V=0), "V >= 1"),
])
def test_walks_that_are_refused(over, fragment):
    assert walk(**over) == BAD and fragment in said()
    assert walk(N=257) == RANGE and walk(V=(1 << 21) + 1) == RANGE and walk(B=1 << 30) == RANGE
    assert walk(p=None, u=None, choices=PTR, N=257) == RANGE


@pytest.mark.parametrize("over,fragment", [
    (dict(B=0), "B >= 1"), (dict(N=0), "N >= 1"), (dict(layers=0), "n_layers"), (dict(held=None), "NULL"), (dict(path=None), "NULL"), (dict(layers=2, stride=4), "layer_stride"),
    (dict(layers=2, stride=-8), "layer_stride"), (dict(layers=2, stride=0), "layer_stride"),
])
def test_kept_paths_that_are_refused(over, fragment):
    assert keep(**over) == BAD and fragment in said()
    assert keep(N=257) == RANGE and keep(B=1 << 20, layers=1 << 10, stride=4096) == RANGE


def test_workspaces():
    n = C.c_size_t()
    need = lambda f, *a: (f(C.byref(cache()), *a, C.byref(n)), n.value)
    # a window that is short is never split, however long the cache is; nor are trees over short caches
    assert need(L.tsd_window_attn_workspace, 1, 1, 4, 1 << 30, 100, 4) == (0, 0)
    assert need(L.tsd_tree_attn_workspace, 1, 20, 4, 100, 0, 0) == (0, 0)
    rc, size = need(L.tsd_window_attn_workspace, 1, 1, 4, 1 << 30, 5000, 4)
    assert rc == 0 and size > 2 * 4 * 65 * 4
    assert need(L.tsd_window_attn_workspace, 1, 1, 4, 5004, 5000, 4) == (rc, size)
    # without a window a call is as large as causal attention's
    for T, m in ((1, 5000), (26, 32768), (256, 3000)):
        causal = need(L.tsd_paged_attn_workspace, 1, T, 4, m)
        assert need(L.tsd_window_attn_workspace, 1, T, 4, m, 1 << 30, 0) == causal == need(L.tsd_tree_attn_workspace, 1, T, 4, m, 0, 0)
    assert L.tsd_window_attn_workspace(C.byref(cache()), 1, 1, 4, 100, 10, 0, None) == BAD
    assert L.tsd_tree_attn_workspace(C.byref(cache()), 1, 1, 4, 100, 10, 0, None) == BAD
    assert L.tsd_token_logprobs_workspace(1000, 1, 32000, 5, C.byref(n)) == 0 and n.value == 0
    for rows_, V, top in ((1, 131072, 5), (1, 1 << 23, 32), (700, 1 << 23, 0)):
        assert L.tsd_token_logprobs_workspace(rows_, 1, V, top, C.byref(n)) == 0 and rows_ * 2 * (24 + 8 * top) <= n.value <= rows_ * 32 * (24 + 8 * top)
    assert L.tsd_token_logprobs_workspace(1, 1, 100, 0, None) == BAD
    assert L.tsd_verify_tree_workspace(3, 20, 32000, tsd.TSD_BF16, C.byref(n)) == 0 and n.value == 0
    assert L.tsd_verify_tree_workspace(3, 20, 131072, tsd.TSD_BF16, C.byref(n)) == 0 and n.value == 3 * 20 * 4
    assert L.tsd_verify_tree_workspace(3, 20, 32000, tsd.TSD_BF16, None) == BAD


@pytest.mark.parametrize("dtype", [tsd.TSD_BF16, tsd.TSD_F32])
@pytest.mark.parametrize("B", [1, 3, 16, 100, 5000])
def test_plans_of_all_sizes(dtype, B):
    # every length, few rows and many: a plan is made, of parts that hold at least a step of keys each
    n, c = C.c_size_t(), cache(dtype=dtype)
    for T in (1, 8, 40, 64, 256):
        for m in [*range(1, 140), 200, 255, 256, 257, 300, 511, 513, 1000, 1025, 2047, 2049, 4095, 5000, 16384, 100000, 1 << 20, 1 << 30]:
            for w, sinks in ((0, 0), (1, 0), (70, 3), (5000, 64), (1 << 30, 1 << 30)):
                for call in ([L.tsd_tree_attn_workspace] if w == 0 else [L.tsd_tree_attn_workspace, L.tsd_window_attn_workspace]):
                    assert call(C.byref(c), B, T, 8, m, w, sinks, C.byref(n)) == 0
                    places = min(m, sinks + w + T) if w else m
                    assert n.value <= (places // 32 + 1) * B * (T * 8 * 65 * 4 + 4 * (T * 2 // 16 + 1) * 8) + 256
                    assert places > 32 or n.value == 0


z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
i32, i64 = torch.int32, torch.int64
ATTN = lambda: [z(2, 3, 4, 64), z(9, 16, 4, 64), z(9, 16, 4, 64), z(2, 4, dtype=i32), z(2, dtype=i32)]
CALLS = {
    "window": lambda *a: tsd.window_attn_static(*(a or ATTN()), 10),
    "tree": lambda *a: tsd.tree_attn_static(*(a or ATTN()), z(2, 3, dtype=i32)),
    "scores": lambda *a: tsd.token_logprobs_static(*(a or [z(2, 3, 50), z(2, 3, dtype=i64)])),
    "walk": lambda *a: tsd.verify_tree_static(*(a or [z(2, 5, dtype=i32), z(2, 5, dtype=i32), z(2, 5, 50), z(2, 5)])),
    "keep": lambda *a: tsd.keep_path_static(*(a or [z(9, 16, 4, 64), z(9, 16, 4, 64), z(2, 4, dtype=i32), z(2, dtype=i32), z(2, 5, dtype=i32)])),
}


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_the_host_and_what_is_no_tensor(name):
    with pytest.raises(ValueError, match="cuda"):
        CALLS[name]()


def test_what_is_no_tensor_and_options():
    q, k, v, table, lens = ATTN()
    for call in (lambda: tsd.window_attn_static([1], k, v, table, lens, 5), lambda: tsd.tree_attn_static(q, k, None, table, lens, z(3, dtype=i32)),
                 lambda: tsd.token_logprobs_static([1.0]), lambda: tsd.verify_tree_static([[1]], z(2, 5, dtype=i32)),
                 lambda: tsd.keep_path_static(k, v, table, lens, [[0]])):
        with pytest.raises(TypeError, match="tensor"):
            call()
    for o in (dict(max_len=0), dict(scale=math.nan)):
        with pytest.raises(ValueError, match=next(iter(o))):
            tsd.window_attn_static(q, k, v, table, lens, 5, **o)
        with pytest.raises(ValueError, match=next(iter(o))):
            tsd.tree_attn_static(q, k, v, table, lens, z(3, dtype=i32), **o)
    with pytest.raises(ValueError, match="window"):
        tsd.tree_attn_static(q, k, v, table, lens, z(3, dtype=i32), window=0)


@pytest.mark.parametrize("name,at", [("window", 0), ("window", 1), ("window", 2), ("tree", 0), ("tree", 1), ("tree", 2), ("scores", 0), ("keep", 0), ("keep", 1)])
def test_refused_while_gradients_are_recorded(name, at):
    args = {"window": ATTN, "tree": ATTN, "scores": lambda: [z(2, 3, 50)],
            "keep": lambda: [z(9, 16, 4, 64), z(9, 16, 4, 64), z(2, 4, dtype=i32), z(2, dtype=i32), z(2, 5, dtype=i32)]}[name]()
    args[at].requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        CALLS[name](*args)
    with torch.no_grad(), pytest.raises(ValueError, match="cuda"):
        CALLS[name](*args)


@pytest.mark.parametrize("name", CALLS)
def test_an_older_extension_says_that_it_is_to_be_built(monkeypatch, name):
    m = types.ModuleType("paper_2511_18191_amd._torch_calls")
    m.bind, m.bind_round, m.paged_attn_static = lambda a: None, lambda *a: None, lambda *a: (0, "out", None)
    monkeypatch.setitem(sys.modules, m.__name__, m)
    monkeypatch.setattr(tsd, "_torch_calls", m, raising=False)
    for n in ("_calls", "_round_calls", "_tree_calls"):
        monkeypatch.setattr(binding, n, None, raising=False)
    with pytest.raises(RuntimeError, match="_torch_calls.so.*build"):
        CALLS[name]()
    assert tsd.paged_attn_static(None, None, None, None, None) == "out"       # what it has goes on working
