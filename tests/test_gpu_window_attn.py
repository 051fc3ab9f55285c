"""window_attn_static against its definition in 64 bits (tests/tree_ref.py), within bounds that count roundings."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import check_attention, paged
from tree_ref import attention

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def inputs(B, T, Hq, Hkv, D, page, dtype, lens, seed=0, order="token", cols=None):
    cols = cols or max(1, -(-max(lens) // page))
    k, v, table = paged(B, cols, page, Hkv, D, dtype, seed, order)
    g = torch.Generator().manual_seed(seed + 1)
    q = (1.5 * torch.randn(B, T, Hq, D, generator=g)).to(dtype).cuda()
    return q, k, v, table, torch.tensor(lens, dtype=torch.int32).cuda()


def run(q, k, v, table, lens, window, sinks=0, **over):
    before = torch.full_like(q, 7.0)
    out, lse = tsd.window_attn_static(q, k, v, table, lens, window, sinks=sinks, out=before.clone(), want_lse=True, **over)
    check_attention(out, lse, attention(q, k, v, table, lens, over.get("n_new"), over.get("scale"), window, sinks), before)
    return out, lse


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (16, 4), (31, 0), (33, 40), (64, 4), (1000, 7), (1 << 30, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,page,lens", [
    (3, 1, 4, 4, 64, 16, [1, 16, 400]),
    (2, 5, 6, 2, 64, 16, [5, 300]),                  # three heads a key head, rows that fill no tile
    (2, 3, 4, 2, 80, 8, [190, 3]),                   # an odd head size, pages smaller than a step
    (1, 2, 2, 1, 256, 16, [170]),
    (1, 3, 2, 2, 24, 1, [77]),                       # a token a page
])
def test_sizes(dtype, window, sinks, B, T, Hq, Hkv, D, page, lens):
    run(*inputs(B, T, Hq, Hkv, D, page, dtype, lens), window, sinks)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 5), (100, 130), (64, 64), (127, 0), (333, 4), (1 << 30, 3)])
@pytest.mark.parametrize("T,Hq,Hkv,D,lens", [(200, 4, 2, 64, [533, 200]), (70, 8, 1, 128, [70, 700]), (130, 2, 2, 80, [131, 600])])
def test_chunks_of_prompts(dtype, window, sinks, T, Hq, Hkv, D, lens):
    run(*inputs(2, T, Hq, Hkv, D, 16, dtype, lens), window, sinks)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 4, 2, 128), (5, 4, 2, 64), (3, 2, 2, 256), (70, 2, 2, 64)])
def test_split_over_a_long_window(dtype, T, Hq, Hkv, D):
    q, k, v, table, lens = inputs(3, T, Hq, Hkv, D, 64, dtype, [6099, 1, 2500])
    for window, sinks in ((3000, 4), (3000, 0), (100, 2000), (5999, 33)):
        out, lse = run(q, k, v, table, lens, window, sinks)
        again = tsd.window_attn_static(q, k, v, table, lens, window, sinks=sinks, out=torch.full_like(q, 7.0), want_lse=True)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])      # the same bits
    for max_len in (1, 100, 1000, 6099, 1 << 20):                             # what the host knows: right whatever it says
        run(q, k, v, table, lens, 3000, 4, max_len=max_len)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [4, 80])
def test_ragged_and_empty(dtype, T):
    # no tokens cached, no new ones, fewer cached than new, counts out of range (clamped)
    q, k, v, table, lens = inputs(6, T, 4, 2, 64, 16, dtype, [0, 20, 3, 1, 170, -5], cols=12)
    for n_new in ([0, 2, 4, 1, 99, 2], [4, -3, 0, 4, 1, 4], None):
        run(q, k, v, table, lens, 9, 2, n_new=None if n_new is None else torch.tensor(n_new, dtype=torch.int32).cuda())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [1, 3, 70])
def test_dropped_pages(dtype, T):
    # pages out of every window are holes, and so may some within be; the same as with them, to the bit
    q, k, v, table, lens = inputs(2, T, 4, 2, 64, 16, dtype, [3000, 900])
    window, sinks = 200, 5
    full = run(q, k, v, table, lens, window, sinks)
    dropped = table.clone()
    for b, n in enumerate(lens.tolist()):
        dropped[b, 1: (n - T - window + 1) // 16] = (-1, k.shape[0] + 5)[b]
    got = run(q, k, v, dropped, lens, window, sinks)
    assert torch.equal(got[0], full[0]) and torch.equal(got[1], full[1])
    dropped[0, 2999 // 16 - 3] = -1
    dropped[:, 0] = -1
    run(q, k, v, dropped, lens, window, sinks)
    out, lse = run(q, k, v, torch.full_like(table, -1), lens, window, sinks)
    assert not out.any() and bool((lse == -math.inf).all())
    run(q, k, v, table[:, :20], lens, window, sinks)          # tokens beyond the table's columns are holes
    run(q, k, v, table[:, :20], lens, 1 << 30, 0)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq,D,order", [(1, 4, 64, "token"), (5, 4, 128, "head"), (20, 4, 80, "head"), (90, 2, 64, "token")])
def test_what_no_row_sees_may_hold_anything(dtype, T, Hq, D, order):
    q, k, v, table, lens = inputs(2, T, Hq, 2, D, 16, dtype, [137, 500], order=order, cols=40)
    window, sinks = 30, 3
    ref = attention(q, k, v, table, lens, window=window, sinks=sinks)
    seen = torch.zeros(k.shape[:2], dtype=torch.bool)
    for b, n in enumerate(lens.tolist()):
        for j in range(n):
            if j < sinks or j > n - T - window:
                seen[int(table[b, j // 16]), j % 16] = True
    for pool, bad in ((k, math.nan), (v, math.nan), (v, math.inf)):
        pool[~seen.cuda()] = bad
        out, lse = tsd.window_attn_static(q, k, v, table, lens, window, sinks=sinks, want_lse=True)
        check_attention(out, lse, ref)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq", [(5, 4), (17, 8), (150, 2)])
def test_a_token_that_is_not_finite_reaches_only_those_that_see_it(dtype, T, Hq):
    q, k, v, table, lens = inputs(2, T, Hq, 2, 64, 16, dtype, [2 * T + 64, 33 + T])
    window, sinks = 3, 2
    ref = attention(q, k, v, table, lens, window=window, sinks=sinks)
    for bad in (math.nan, math.inf, -math.inf):
        for pool in (k, v):
            kept = pool.clone()
            sees = torch.zeros(2, T, dtype=torch.bool)
            for b, n in enumerate(lens.tolist()):
                j = n - T + T // 2                            # some token in the middle
                pool[int(table[b, j // 16]), j % 16, :, 3] = bad
                sees[b, T // 2: T // 2 + window] = True
            out = tsd.window_attn_static(q, k, v, table, lens, window, sinks=sinks)
            pool.copy_(kept)
            off = (out.double().cpu() - ref[0]).abs()
            assert bool((off[~sees] <= ref[2][~sees]).all())
            if pool is v or math.isnan(bad):
                assert not bool(torch.isfinite(out.cpu()[sees]).all(-1).any())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [8, 32, 72, 80, 88, 96, 104, 120, 128, 136, 160, 192, 200, 248, 256])
def test_head_sizes(dtype, D):
    # few rows and many, one key head for three query heads
    for T, lens in ((2, [50, 300]), (45, [45, 400])):
        run(*inputs(2, T, 3, 1, D, 16, dtype, lens), 60, 4)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_a_window_as_long_as_the_sequence_is_causal_attention(dtype):
    for T, lens in ((3, [900, 77]), (100, [500, 100])):
        q, k, v, table, lens = inputs(2, T, 4, 2, 64, 16, dtype, lens)
        a = tsd.window_attn_static(q, k, v, table, lens, 1 << 20, want_lse=True)
        b = tsd.paged_attn_static(q, k, v, table, lens, want_lse=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [BF, FP])
def test_strides_and_out_in_place(dtype):
    B, T, Hq, Hkv, D, page = 3, 4, 4, 2, 64, 16
    g = torch.Generator().manual_seed(3)
    fused = torch.randn(B, T, Hq + 2 * Hkv, D, generator=g).to(dtype).cuda()
    both = torch.randn(20, 2, Hkv, page, D, generator=g).to(dtype).cuda()
    k, v = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    table = torch.randperm(20, generator=g)[:18].to(torch.int32).view(3, 6).cuda()[:, 1:5]
    lens = torch.tensor([64, 1, 50], dtype=torch.int32).cuda()
    wide = torch.full((B, T, Hq, 2 * D), 7.0, dtype=dtype).cuda()
    q, out = fused[:, :, :Hq], wide[..., :D]
    tsd.window_attn_static(q, k, v, table, lens, 20, sinks=2, out=out)
    ref = attention(q, k, v, table, lens, window=20, sinks=2)
    check_attention(out, None, ref)
    assert bool((wide[..., D:] == 7.0).all())
    x = q.contiguous()
    tsd.window_attn_static(x, k, v, table, lens, 20, sinks=2, out=x)
    assert torch.equal(x, out)
    run(q, k, v, table, lens, 20, 2, scale=-0.5)
    run(q, k, v, table, lens, 20, 2, scale=0.0)


@pytest.mark.parametrize("T,lens", [(3, [3000, 2100]), (2, [900, 700]), (150, [900, 700])])
def test_streams_and_replayed_graphs(T, lens):
    # two captured calls over one cache, replayed on two streams while eager calls run; lengths move on between the replays
    q, k, v, table, lens = inputs(2, T, 4, 2, 64, 16, BF, lens, cols=200)
    outs = [torch.zeros_like(q) for _ in range(2)]
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    for out, s in zip(outs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                tsd.window_attn_static(q, k, v, table, lens, 800, sinks=4, out=out)
            graphs.append(g)
    torch.cuda.synchronize()
    for step in range(4):
        lens += 13 * step + 1
        torch.cuda.synchronize()
        want = tsd.window_attn_static(q, k, v, table, lens, 800, sinks=4)
        for out, s, g in zip(outs, streams, graphs):
            out.zero_()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    check_attention(want, None, attention(q, k, v, table, lens, window=800, sinks=4))
