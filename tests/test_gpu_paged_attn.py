"""paged_attn_static against its definition in 64 bits (tests/round_ref.py), within bounds that count roundings."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import attention, check_attention, paged

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def inputs(B, T, Hq, Hkv, D, page, dtype, lens, seed=0, order="token", cols=None):
    cols = cols or max(1, -(-max(lens) // page))
    k, v, table = paged(B, cols, page, Hkv, D, dtype, seed, order)
    g = torch.Generator().manual_seed(seed + 1)
    q = (1.5 * torch.randn(B, T, Hq, D, generator=g)).to(dtype).cuda()
    return q, k, v, table, torch.tensor(lens, dtype=torch.int32).cuda()


def run(q, k, v, table, lens, **over):
    before = torch.full_like(q, 7.0)
    out, lse = tsd.paged_attn_static(q, k, v, table, lens, out=before.clone(), want_lse=True, **over)
    n_new, scale = over.get("n_new"), over.get("scale")
    check_attention(out, lse, attention(q, k, v, table, lens, n_new, scale), before)
    return out, lse


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,page,lens", [
    (1, 1, 1, 1, 64, 16, [1]),
    (3, 1, 4, 4, 64, 16, [1, 16, 17]),
    (4, 1, 8, 1, 128, 32, [31, 32, 33, 64]),
    (3, 5, 6, 2, 64, 16, [5, 61, 129]),              # three heads a key head, rows that fill no tile
    (2, 17, 4, 4, 128, 64, [17, 200]),               # K = 16 proposals
    (2, 7, 16, 2, 96, 16, [300, 7]),                 # 56 rows a key head
    (2, 3, 4, 2, 80, 8, [90, 3]),                    # an odd head size, pages smaller than a step
    (2, 2, 3, 3, 8, 1, [40, 2]),                     # the smallest head, a token a page
    (2, 2, 2, 1, 256, 16, [70, 33]),
    (1, 9, 6, 1, 200, 1024, [1500]),
    (1, 4, 2, 1, 40, 2, [700]),
])
def test_sizes(dtype, B, T, Hq, Hkv, D, page, lens):
    run(*inputs(B, T, Hq, Hkv, D, page, dtype, lens))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq,Hkv,D", [(1, 4, 2, 128), (5, 4, 2, 64), (3, 2, 2, 256)])
def test_split_over_a_long_cache(dtype, T, Hq, Hkv, D):
    q, k, v, table, lens = inputs(3, T, Hq, Hkv, D, 64, dtype, [4099, 1, 2500])
    out, lse = run(q, k, v, table, lens)
    again = tsd.paged_attn_static(q, k, v, table, lens, out=torch.full_like(q, 7.0), want_lse=True)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])          # the same bits
    for max_len in (100, 1000, 4099, 1 << 20):                                # what the host knows: right whatever it says
        run(q, k, v, table, lens, max_len=max_len)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq,Hkv,D,lens", [(200, 4, 2, 64, [333, 200]), (65, 8, 1, 128, [65, 700]), (130, 2, 2, 80, [131, 400])])
def test_chunks_of_prompts(dtype, T, Hq, Hkv, D, lens):
    run(*inputs(2, T, Hq, Hkv, D, 16, dtype, lens))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_ragged_and_empty(dtype):
    # no tokens cached, no new ones, fewer cached than new, counts out of range (clamped)
    lens = [0, 20, 3, 1, 70, -5]
    q, k, v, table, lens = inputs(6, 4, 4, 2, 64, 16, dtype, lens, cols=5)
    run(q, k, v, table, lens, n_new=torch.tensor([0, 2, 4, 1, 99, 2], dtype=torch.int32).cuda())
    run(q, k, v, table, lens, n_new=torch.tensor([4, -3, 0, 4, 1, 4], dtype=torch.int32).cuda())
    run(q, k, v, table, lens)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("long", [False, True])
def test_holes_and_lengths_beyond_the_table(dtype, long):
    lens = [3000, 2900] if long else [60, 45]
    q, k, v, table, lens = inputs(2, 3, 4, 2, 64, 16, dtype, lens)
    table[0, 1], table[1, 0], table[1, 2], table[0, -1] = -1, k.shape[0], 2 ** 31 - 1, -2 ** 31
    run(q, k, v, table, lens)
    run(q, k, v, table[:, :2], lens)                          # the rest of the sequence has no pages: holes
    table[:] = -1
    out, lse = run(q, k, v, table, lens)                      # nothing to see at all
    assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,D,order", [(1, 64, "token"), (5, 128, "head"), (20, 80, "head")])
def test_what_no_row_sees_may_hold_anything(dtype, T, D, order):
    lens = [37, 500]
    q, k, v, table, lens = inputs(2, T, 4, 2, D, 16, dtype, lens, order=order, cols=40)
    ref = attention(q, k, v, table, lens)
    seen = torch.zeros(k.shape[:2], dtype=torch.bool)
    for b, n in enumerate(lens.tolist()):
        for j in range(n):
            seen[int(table[b, j // 16]), j % 16] = True
    for pool, bad in ((k, math.nan), (v, math.nan), (v, math.inf)):
        pool[~seen.cuda()] = bad
        out, lse = tsd.paged_attn_static(q, k, v, table, lens, want_lse=True)
        check_attention(out, lse, ref)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("T,Hq", [(5, 4), (17, 8)])
def test_a_later_token_that_is_not_finite_reaches_no_earlier_one(dtype, T, Hq):
    lens = [64, 33 + T]
    q, k, v, table, lens = inputs(2, T, Hq, 2, 64, 16, dtype, lens)
    ref = attention(q, k, v, table, lens)
    for bad in (math.nan, math.inf, -math.inf):
        for pool in (k, v):
            kept = pool.clone()
            for b, n in enumerate(lens.tolist()):
                j = n - 2                                     # the last token but one
                pool[int(table[b, j // 16]), j % 16, :, 3] = bad
            out = tsd.paged_attn_static(q, k, v, table, lens)
            pool.copy_(kept)
            early = torch.zeros(2, T, dtype=torch.bool)
            early[:, : T - 2] = True
            off = (out.double().cpu() - ref[0]).abs()
            assert bool((off[early] <= ref[2][early]).all())
            if pool is v or math.isnan(bad):
                assert not bool(torch.isfinite(out[:, T - 1]).all())          # and it does reach those that see it


def test_scores_of_minus_infinity():
    # keys of -inf where the query is positive: weight 0; a row with nothing else counts as empty
    q, k, v, table, lens = inputs(1, 1, 2, 2, 64, 16, FP, [20])
    q[..., 5] = 1.0
    at = lambda j: (int(table[0, j // 16]), j % 16)
    for j in range(3, 20):
        k[at(j)][:, 5] = -math.inf
    short = torch.tensor([3], dtype=torch.int32).cuda()
    ref = attention(q, k, v, table, short)
    out, lse = tsd.paged_attn_static(q, k, v, table, lens, want_lse=True)
    check_attention(out, lse, ref)
    for j in range(3):
        k[at(j)][:, 5] = -math.inf
    out, lse = tsd.paged_attn_static(q, k, v, table, lens, want_lse=True)
    assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF, FP])
def test_strides(dtype):
    # queries inside a fused projection, outputs inside a wider tensor, a cache with keys and values of a page side by side, heads outside tokens
    B, T, Hq, Hkv, D, page = 3, 4, 4, 2, 64, 16
    g = torch.Generator().manual_seed(3)
    fused = torch.randn(B, T, Hq + 2 * Hkv, D, generator=g).to(dtype).cuda()
    both = torch.randn(20, 2, Hkv, page, D, generator=g).to(dtype).cuda()
    k, v = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    wide_table = torch.randperm(20, generator=g)[:18].to(torch.int32).view(3, 6).cuda()
    table, lens = wide_table[:, 1:5], torch.tensor([64, 1, 50], dtype=torch.int32).cuda()
    wide = torch.full((B, T, Hq, 2 * D), 7.0, dtype=dtype).cuda()
    q, out = fused[:, :, :Hq], wide[..., :D]
    assert tsd.paged_attn_static(q, k, v, table, lens, out=out) is not None
    check_attention(out, None, attention(q, k, v, table, lens))
    assert bool((wide[..., D:] == 7.0).all())
    rows = torch.randn(T, B, Hq, D, generator=g).to(dtype).cuda().transpose(0, 1)          # tokens outside sequences
    run(rows, k, v, table, lens)
    one = torch.randn(B, 1, 1, D, generator=g).to(dtype).cuda().expand(B, T, Hq, D)        # the same query everywhere
    run(one, k, v, table, lens, scale=-0.5)
    run(one, k, v, table, lens, scale=0.0)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_offsets_beyond_32_bits(dtype):
    page, Hkv, D = 64, 8, 128
    n = (1 << 32) // (page * Hkv * D) + 40          # element offsets pass 2^32
    if torch.cuda.mem_get_info()[0] < 3 * n * page * Hkv * D * 4:
        pytest.skip("needs some 50 GB of device memory")
    k, v = (torch.empty(n, page, Hkv, D, dtype=dtype, device="cuda") for _ in range(2))
    pages = [n - 1, 5, n - 30, n // 2 + 1, 0]
    small = torch.randn(2, len(pages), page, Hkv, D, generator=torch.Generator().manual_seed(4)).to(dtype).cuda()
    for i, at in enumerate(pages):
        k[at], v[at] = small[0, i], small[1, i]
    q = torch.randn(1, 2, 8, D, generator=torch.Generator().manual_seed(5)).to(dtype).cuda()
    lens = torch.tensor([300], dtype=torch.int32).cuda()
    out, lse = tsd.paged_attn_static(q, k, v, torch.tensor([pages], dtype=torch.int32).cuda(), lens, want_lse=True)
    check_attention(out, lse, attention(q, small[0], small[1], torch.arange(5, dtype=torch.int32)[None], lens))


def test_many_sequences():
    B = 700
    lens = [(7 * i) % 90 + 1 for i in range(B)]
    run(*inputs(B, 2, 2, 1, 64, 16, BF, lens))


def test_streams_and_replayed_graphs():
    # two captured calls over one cache, replayed on two streams while eager calls run; lengths move on between the replays
    q, k, v, table, lens = inputs(2, 3, 4, 2, 64, 16, BF, [3000, 2100], cols=200)
    outs = [torch.zeros_like(q) for _ in range(2)]
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    for out, s in zip(outs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            tsd.paged_attn_static(q, k, v, table, lens, out=out)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                tsd.paged_attn_static(q, k, v, table, lens, out=out)
            graphs.append(g)
    torch.cuda.synchronize()
    for step in range(4):
        lens += 13 * step + 1
        torch.cuda.synchronize()
        want = tsd.paged_attn_static(q, k, v, table, lens)
        for out, s, g in zip(outs, streams, graphs):
            out.zero_()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    check_attention(want, None, attention(q, k, v, table, lens))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,lens", [(2, 2, 4, 2, 64, [1000, 700]), (3, 1, 2, 1, 128, [1500, 3, 900]), (1, 70, 2, 2, 64, [600])])
def test_parts_joined_by_the_last_workgroup(dtype, B, T, Hq, Hkv, D, lens):
    # small joins take no second launch: alone, again in the same memory, replayed, and on two streams at once
    q, k, v, table, lens = inputs(B, T, Hq, Hkv, D, 16, dtype, lens, cols=100)
    run(q, k, v, table, lens)
    outs, graphs, streams = [torch.zeros_like(q) for _ in range(2)], [], [torch.cuda.Stream() for _ in range(2)]
    for out, s in zip(outs, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                tsd.paged_attn_static(q, k, v, table, lens, out=out)
                q_next = out * 2
                tsd.paged_attn_static(q_next, k, v, table, lens, out=out)
            graphs.append((g, q_next))
    for step in range(20):
        q.normal_()
        torch.cuda.synchronize()
        want = tsd.paged_attn_static(tsd.paged_attn_static(q, k, v, table, lens) * 2, k, v, table, lens)
        for s, (g, _) in zip(streams, graphs):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    check_attention(want, None, attention(tsd.paged_attn_static(q, k, v, table, lens) * 2, k, v, table, lens))


@pytest.mark.parametrize("rows", [33, 40, 64, 65, 128, 129])
def test_row_tiles(rows):
    # wide heads and workgroups enough: tiles of 128 rows, some of whose wavefronts have none
    B, Hkv = 70, 1
    run(*inputs(B, rows, Hkv, Hkv, 128, 16, BF, [130 + (11 * i) % 90 for i in range(B)]))


def test_maxima_that_rise_slowly_and_at_once():
    # a row's later keys outweigh its earlier ones by a little at a time, or by far: the running maximum may lag behind, the result may not
    B, T, D, n = 2, 130, 128, 700
    q, k, v, table, lens = inputs(B, T, 1, 1, D, 16, BF, [n, n])
    q[:] = 0
    q[..., 0] = 8.0
    for b in range(B):
        for j in range(n):
            at = int(table[b, j // 16]), j % 16
            k[at] = 0
            k[at][0, 0] = j * 0.02 if b == 0 else (0.0 if j < 400 else 60.0)
    for scale in (None, 1.0, -1.0):
        run(q, k, v, table, lens, scale=scale)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [8, 24, 32, 72, 96, 120, 128, 136, 192, 256])
def test_head_sizes(dtype, D):
    # few rows and many, one key head for three query heads
    for T, lens in ((2, [50, 300]), (45, [45, 200])):
        run(*inputs(2, T, 3, 1, D, 16, dtype, lens))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,T,D,lens", [(2, 3, 64, [70, 20]), (2, 2, 64, [900, 700]), (1, 5, 128, [9000]), (1, 200, 128, [700])])
def test_out_may_be_q(dtype, B, T, D, lens):
    # whole, joined by the last workgroup, joined by a second launch, many rows
    q, k, v, table, lens = inputs(B, T, 4, 2, D, 16, dtype, lens)
    want = tsd.paged_attn_static(q, k, v, table, lens)
    got = q.clone()
    assert tsd.paged_attn_static(got, k, v, table, lens, out=got) is not None
    assert torch.equal(got, want)
