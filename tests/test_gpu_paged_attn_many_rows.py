"""paged_attn_static with so many rows a key head that the kernel for prompts takes them: its own masks and loads, where a sequence has no keys or no new
tokens, pages are missing, tokens are not finite, tensors lie otherwise.  Against the definition in 64 bits (tests/round_ref.py)."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import attention, check_attention
from test_gpu_paged_attn import inputs, run

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
# T, Hq, Hkv, D: 80 rows a key head of each width, 300 rows (three tiles) of an odd width, 70 of the smallest
SHAPES = [(40, 4, 2, 64), (40, 4, 2, 128), (150, 2, 1, 80), (70, 1, 1, 8)]
i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("long", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,D", SHAPES)
def test_ragged_and_empty(T, Hq, Hkv, D, long):
    # no tokens cached, no new ones, fewer cached than new, counts out of range (clamped), tiles and wavefronts without rows
    lens = [0, 20, 3, 1, 2100 if long else 130, -5, T + 2]
    q, k, v, table, lens = inputs(len(lens), T, Hq, Hkv, D, 16, BF, lens, cols=140 if long else 11)
    run(q, k, v, table, lens, n_new=i32([0, 2, T, 1, T + 59, 2, T // 2]))
    run(q, k, v, table, lens, n_new=i32([T, -3, 0, T, 1, T, 33]))
    run(q, k, v, table, lens)


@pytest.mark.parametrize("n", [100, 1500])
@pytest.mark.parametrize("T,Hq,Hkv,D", SHAPES)
def test_holes_and_lengths_beyond_the_table(T, Hq, Hkv, D, n):
    q, k, v, table, lens = inputs(2, T, Hq, Hkv, D, 16, BF, [n, n - 13])
    table[0, 1], table[0, 3], table[0, -1] = -1, k.shape[0], 2 ** 31 - 1          # inside tiles of 64 keys, and at the end
    table[1, :4] = -2 ** 31                                                       # a whole tile, the first
    run(q, k, v, table, lens)
    run(q, k, v, table, lens, n_new=i32([T, 3]))
    run(q, k, v, table[:, :5], lens)                                              # the rest of the sequences has no pages
    run(q, k, v, table, lens + 70)                                                # longer than the table
    run(q, k, v, table[:, :1], lens)
    table[:] = -1
    out, lse = run(q, k, v, table, lens)                                          # nothing to see at all
    assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("order", ["token", "head"])
@pytest.mark.parametrize("T,Hq,Hkv,D", SHAPES)
def test_what_no_row_sees_may_hold_anything(T, Hq, Hkv, D, order):
    lens = [T - 3, 700]                      # (rows of the first that see no key at all)
    q, k, v, table, lens = inputs(2, T, Hq, Hkv, D, 16, BF, lens, order=order, cols=50)
    ref = attention(q, k, v, table, lens)
    seen = torch.zeros(k.shape[:2], dtype=torch.bool)
    for b, n in enumerate(lens.tolist()):
        for j in range(n):
            seen[int(table[b, j // 16]), j % 16] = True
    for pool, bad in ((k, math.nan), (v, math.nan), (k, -math.inf), (v, math.inf)):
        pool[~seen.cuda()] = bad
        out, lse = tsd.paged_attn_static(q, k, v, table, lens, want_lse=True)
        check_attention(out, lse, ref)


@pytest.mark.parametrize("back", [2, 20])
@pytest.mark.parametrize("T,Hq,Hkv,D", SHAPES)
def test_a_later_token_that_is_not_finite_reaches_no_earlier_one(T, Hq, Hkv, D, back):
    lens = [T, 333 + T]
    q, k, v, table, lens = inputs(2, T, Hq, Hkv, D, 16, BF, lens)
    ref = attention(q, k, v, table, lens)
    for bad in (math.nan, math.inf, -math.inf):
        for pool in (k, v):
            kept = pool.clone()
            for b, n in enumerate(lens.tolist()):
                j = n - back                 # the token that the last back - 1 tokens see, and itself
                pool[int(table[b, j // 16]), j % 16, :, 3] = bad
            out = tsd.paged_attn_static(q, k, v, table, lens)
            pool.copy_(kept)
            early = torch.zeros(2, T, dtype=torch.bool)
            early[:, : T - back] = True
            off = (out.double().cpu() - ref[0]).abs()
            assert bool((off[early] <= ref[2][early]).all())
            if pool is v:
                assert not bool(torch.isfinite(out[:, T - back:, :, 3]).any())       # it reaches all that see it, in its dim
            elif math.isnan(bad):
                assert not bool(torch.isfinite(out[:, T - back:]).any())


@pytest.mark.parametrize("T,Hq,Hkv,D", SHAPES)
def test_scores_of_minus_infinity(T, Hq, Hkv, D):
    # keys of -inf where the queries are positive weigh nothing: a first tile of them, others between, and at last nothing else
    n = T + 150
    q, k, v, table, lens = inputs(1, T, Hq, Hkv, D, 1, BF, [n])
    q[..., 5] = 1.0
    without = table.clone()                  # (a page a token: to the definition these keys are holes)
    for j in [*range(70), 100, 101, n - 3]:
        k[int(table[0, j])][..., 5] = -math.inf
        without[0, j] = -1
    for lens, n_new in ((lens, None), (lens, i32([9])), (i32([T + 60]), None)):        # (of the last, the first rows see such keys only)
        before = torch.full_like(q, 7.0)
        out, lse = tsd.paged_attn_static(q, k, v, table, lens, n_new=n_new, out=before.clone(), want_lse=True)
        check_attention(out, lse, attention(q, k, v, without, lens, n_new), before)
    k[..., 5] = -math.inf
    out, lse = tsd.paged_attn_static(q, k, v, table, lens, want_lse=True)
    assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("D", [64, 128, 80])
def test_strides(D):
    # queries inside a fused projection, outputs inside a wider tensor, keys and values of a page side by side, heads outside tokens
    B, T, Hq, Hkv, page = 3, 45, 4, 2, 16
    g = torch.Generator().manual_seed(3)
    fused = torch.randn(B, T, Hq + 2 * Hkv, D, generator=g).to(BF).cuda()
    both = torch.randn(50, 2, Hkv, page, D, generator=g).to(BF).cuda()
    k, v = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    wide_table = torch.randperm(50, generator=g)[:48].to(torch.int32).view(3, 16).cuda()
    table, lens, n_new = wide_table[:, 1:15], i32([224, 1, 150]), i32([45, 1, 20])
    wide = torch.full((B, T, Hq, 2 * D), 7.0, dtype=BF).cuda()
    q, out = fused[:, :, :Hq], wide[..., :D]
    tsd.paged_attn_static(q, k, v, table, lens, n_new=n_new, out=out)
    check_attention(out, None, attention(q, k, v, table, lens, n_new), torch.full_like(out, 7.0))
    assert bool((wide[..., D:] == 7.0).all())
    rows = torch.randn(T, B, Hq, D, generator=g).to(BF).cuda().transpose(0, 1)             # tokens outside sequences
    run(rows, k, v, table, lens)
    one = torch.randn(B, 1, 1, D, generator=g).to(BF).cuda().expand(B, T, Hq, D)           # the same query everywhere
    for scale in (-0.5, 0.0, 2.0):
        run(one, k, v, table, lens, scale=scale, n_new=n_new)
