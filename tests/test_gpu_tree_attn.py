"""tree_attn_static against its definition in 64 bits (tests/tree_ref.py), within bounds that count roundings."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import check_attention
from test_gpu_window_attn import BF, FP, inputs
from tree_ref import ALL, attention, lines, random_tree

pytestmark = pytest.mark.gpu


def run(q, k, v, table, lens, parents, window=None, sinks=0, **over):
    before = torch.full_like(q, 7.0)
    out, lse = tsd.tree_attn_static(q, k, v, table, lens, parents.cuda(), window=window, sinks=sinks, out=before.clone(), want_lse=True, **over)
    check_attention(out, lse, attention(q, k, v, table, lens, over.get("n_new"), over.get("scale"), window or ALL, sinks, parents), before)
    return out, lse


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("window,sinks", [(None, 0), (1, 0), (3, 2), (40, 4), (300, 30)])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,page,lens", [
    (2, 1, 4, 4, 64, 16, [1, 90]),
    (3, 5, 6, 2, 64, 16, [5, 300, 64]),              # three heads a key head
    (2, 26, 4, 1, 128, 64, [26, 200]),               # 104 rows of one key head
    (2, 17, 3, 3, 80, 8, [190, 20]),                 # an odd head size, pages smaller than a step
    (1, 33, 2, 1, 256, 16, [170]),
    (1, 64, 2, 2, 64, 16, [333]),
    (2, 65, 2, 1, 96, 16, [70, 65]),
    (1, 200, 2, 2, 32, 32, [777]),
    (1, 256, 1, 1, 64, 1, [256]),                    # the most nodes, a token a page, nothing before the tree
])
def test_sizes(dtype, window, sinks, B, T, Hq, Hkv, D, page, lens):
    run(*inputs(B, T, Hq, Hkv, D, page, dtype, lens), random_tree(B, T, T), window, sinks)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,lens", [(7, [100, 7]), (40, [500, 45]), (130, [300, 130])])
def test_shapes_of_trees(dtype, T, lens):
    q, k, v, table, lens = inputs(2, T, 4, 2, 64, 16, dtype, lens)
    star = torch.zeros(2, T, dtype=torch.int32)
    star[:, 0] = -1
    for parents in (star, torch.full((2, T), -1, dtype=torch.int32), random_tree(2, T, 1, roots=4), random_tree(2, T, 2, reach=300)):
        run(q, k, v, table, lens, parents)
        run(q, k, v, table, lens, parents, 2, 1)
    one = random_tree(1, T, 3)[0]                             # the same tree in every sequence
    a, b = run(q, k, v, table, lens, one), run(q, k, v, table, lens, one.expand(2, T).contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,lens", [(1, [40, 700]), (6, [900, 77]), (100, [500, 100])])
def test_a_chain_is_causal_attention(dtype, T, lens):
    q, k, v, table, lens = inputs(2, T, 4, 2, 64, 16, dtype, lens)
    out, lse = run(q, k, v, table, lens, random_tree(2, T, 0, chain=True))
    ref = attention(q, k, v, table, lens)
    check_attention(out, lse, ref)
    out, lse = run(q, k, v, table, lens, random_tree(2, T, 0, chain=True), 50, 3)
    check_attention(out, lse, attention(q, k, v, table, lens, window=50, sinks=3))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [9, 90])
def test_entries_that_name_no_earlier_node(dtype, T):
    q, k, v, table, lens = inputs(3, T, 4, 2, 64, 16, dtype, [100, 300, T])
    parents = random_tree(3, T, 5)
    parents[0, 3], parents[0, 4], parents[1, 2], parents[2, 5], parents[2, 0], parents[1, 0] = 3, T - 1, 2 ** 31 - 1, -2 ** 31, 4, 1 << 20
    run(q, k, v, table, lens, parents)
    run(q, k, v, table, lens, parents, 2, 0)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 4, 2, 128), (5, 4, 2, 64), (16, 2, 2, 256), (70, 2, 2, 64)])
def test_split_over_a_long_cache(dtype, T, Hq, Hkv, D):
    q, k, v, table, lens = inputs(3, T, Hq, Hkv, D, 64, dtype, [4099, T, 2500])
    parents = random_tree(3, T, 6)
    out, lse = run(q, k, v, table, lens, parents)
    again = tsd.tree_attn_static(q, k, v, table, lens, parents.cuda(), out=torch.full_like(q, 7.0), want_lse=True)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])          # the same bits
    for max_len in (1, 100, 1000, 4099, 1 << 20):
        run(q, k, v, table, lens, parents, max_len=max_len)
        run(q, k, v, table, lens, parents, 2000, 9, max_len=max_len)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [4, 80])
def test_ragged_and_empty(dtype, T):
    # no tokens cached, no new ones, fewer cached than new, counts out of range (clamped)
    q, k, v, table, lens = inputs(6, T, 4, 2, 64, 16, dtype, [0, 20, 3, 1, 170, -5], cols=12)
    parents = random_tree(6, T, 7)
    for n_new in ([0, 2, 4, 1, 99, 2], [4, -3, 0, 4, 1, 4], None):
        n = None if n_new is None else torch.tensor(n_new, dtype=torch.int32).cuda()
        run(q, k, v, table, lens, parents, n_new=n)
        run(q, k, v, table, lens, parents, 3, 2, n_new=n)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T", [5, 70])
def test_holes(dtype, T):
    q, k, v, table, lens = inputs(2, T, 4, 2, 64, 16, dtype, [3000, 290])
    parents = random_tree(2, T, 8)
    table[0, 1], table[1, 0], table[1, 2], table[0, -1] = -1, k.shape[0], 2 ** 31 - 1, -2 ** 31
    run(q, k, v, table, lens, parents)
    run(q, k, v, table, lens, parents, 500, 3)
    run(q, k, v, table[:, :7], lens, parents)
    out, lse = run(q, k, v, torch.full_like(table, -1), lens, parents)
    assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq", [(7, 4), (17, 8), (100, 2)])
def test_a_node_that_is_not_finite_reaches_only_its_line(dtype, T, Hq):
    q, k, v, table, lens = inputs(2, T, Hq, 2, 64, 16, dtype, [T + 64, 33 + T])
    parents = random_tree(2, T, 9)
    ref = attention(q, k, v, table, lens, parents=parents)
    node = T // 2
    sees = torch.stack([lines(parents[b], T)[1][:, node] for b in range(2)])
    for bad in (math.nan, math.inf, -math.inf):
        for pool in (k, v):
            kept = pool.clone()
            for b, n in enumerate(lens.tolist()):
                j = n - T + node
                pool[int(table[b, j // 16]), j % 16, :, 3] = bad
            out = tsd.tree_attn_static(q, k, v, table, lens, parents.cuda())
            pool.copy_(kept)
            off = (out.double().cpu() - ref[0]).abs()
            assert bool((off[~sees] <= ref[2][~sees]).all())
            if pool is v or math.isnan(bad):
                assert not bool(torch.isfinite(out.cpu()[sees]).all(-1).any())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [8, 32, 72, 80, 88, 96, 104, 120, 128, 136, 160, 192, 200, 248, 256])
def test_head_sizes(dtype, D):
    for T, lens in ((3, [50, 300]), (45, [45, 200])):
        run(*inputs(2, T, 3, 1, D, 16, dtype, lens), random_tree(2, T, D))


@pytest.mark.parametrize("T,lens", [(5, [3000, 2100]), (2, [900, 700]), (60, [900, 700])])
def test_streams_and_replayed_graphs(T, lens):
    # two captured calls over one cache, replayed on two streams while eager calls run; lengths and trees change between the replays
    q, k, v, table, lens = inputs(2, T, 4, 2, 64, 16, BF, lens, cols=200)
    parents = random_tree(2, T, 0).cuda()
    outs = [torch.zeros_like(q) for _ in range(2)]
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    for out, s in zip(outs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                tsd.tree_attn_static(q, k, v, table, lens, parents, out=out)
            graphs.append(g)
    torch.cuda.synchronize()
    for step in range(4):
        lens += 13 * step + 1
        parents.copy_(random_tree(2, T, step))
        torch.cuda.synchronize()
        want = tsd.tree_attn_static(q, k, v, table, lens, parents)
        for out, s, g in zip(outs, streams, graphs):
            out.zero_()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    check_attention(want, None, attention(q, k, v, table, lens, parents=parents))
