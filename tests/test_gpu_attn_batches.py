"""tree_attn_static and window_attn_static on batches as they are served: the plans that only many sequences and key heads reach (several row tiles of a tree over chunks
alike, chunks by the workgroups there are, split windows), against the definition in 64 bits, a sequence at a time on the device."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import F32, HALF
from tree_ref import ALL, random_tree, sight

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def inputs(B, T, Hq, Hkv, D, dtype, lens, page=64, n_pages=300, seed=0):
    """Sequences share the pool's pages: nothing is written."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, v = (torch.randn(n_pages, page, Hkv, D, generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.randint(0, n_pages, (B, -(-max(lens) // page)), generator=g, device="cuda").to(torch.int32)
    q = (1.5 * torch.randn(B, T, Hq, D, generator=g, device="cuda")).to(dtype)
    return q, k, v, table, torch.tensor(lens, dtype=torch.int32).cuda()


def check(out, lse, before, q, k_pool, v_pool, table, lens, n_new, window, sinks, parents):
    """As tree_ref.attention says it, with its bounds."""
    B, T, Hq, D = q.shape
    n_pages, page, Hkv, _ = k_pool.shape
    G, scale, half = Hq // Hkv, 1 / math.sqrt(D), HALF[q.dtype]
    rounded = half if q.dtype == BF else 0.0
    for b, length in enumerate(lens.tolist()):
        n = min(max(int(n_new[b]), 0), T)
        assert torch.equal(out[b, n:], before[b, n:]), b
        if not n:
            continue
        sees = sight(length, n, window, sinks, None if parents is None else parents[b]).cuda()
        slots = torch.arange(sees.shape[1], device="cuda")
        pages = table[b, slots // page].long()
        there = sees.any(0) & (pages >= 0) & (pages < n_pages)
        sees, slots, pages = sees[:, there], slots[there], pages[there]
        keys = k_pool[pages, slots % page].double().transpose(0, 1).contiguous()             # [Hkv, m, D]
        vals = v_pool[pages, slots % page].double().transpose(0, 1).contiguous()
        x = q[b, :n].double().view(n, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * n, D).contiguous()
        back = lambda y: y.view(Hkv, G, n, -1).permute(2, 0, 1, 3).reshape(n, Hq, -1)
        kt = keys.transpose(1, 2).contiguous()
        s, mag = torch.bmm(x, kt) * scale, torch.bmm(x.abs(), kt.abs()) * scale
        mine = sees.repeat(G, 1)[None]
        s = torch.where(mine, s, -math.inf)
        top = s.amax(2, keepdim=True)
        assert bool((top > -math.inf).all())                                                 # (every row here sees a key)
        w = torch.exp(s - top)
        total = w.sum(2, keepdim=True)
        want_lse, w = top + torch.log(total), w / total
        want, mass = torch.bmm(w, vals), torch.bmm(w, vals.abs())
        d = torch.where(mine, (D + 8) * F32 * mag + 4 * F32 * s.abs(), 0.0).amax(2, keepdim=True)
        rel = 2 * d + 4 * F32 + (mine.sum(2, keepdim=True) + 40) * F32 + rounded
        tol = (mass + want.abs()) * rel * 1.05 + half * want.abs()
        off = (out[b, :n].double() - back(want)).abs()
        assert bool((off <= back(tol)).all()), (b, float((off / back(tol)).max()))
        off, room = (lse[b, :n].double()[..., None] - back(want_lse)).abs(), back(rel + 4 * F32 * want_lse.abs())
        assert bool((off <= room).all()), (b, float((off / room).max()))


def run(q, k, v, table, lens, n_new, window=None, sinks=0, parents=None, **over):
    before = torch.full_like(q, 7.0)
    call = lambda: (tsd.window_attn_static(q, k, v, table, lens, window, sinks=sinks, n_new=n_new, out=before.clone(), want_lse=True, **over) if parents is None else
                    tsd.tree_attn_static(q, k, v, table, lens, parents.cuda(), window=window, sinks=sinks, n_new=n_new, out=before.clone(), want_lse=True, **over))
    (out, lse), again = call(), call()
    check(out, lse, before, q, k, v, table, lens, n_new, window or ALL, sinks, parents)
    for b, n in enumerate(n_new.tolist()):
        n = min(max(n, 0), q.shape[1])
        assert torch.equal(out[b], again[0][b]) and torch.equal(lse[b, :n], again[1][b, :n])    # the same bits


def ragged(B, T, least, most, seed):
    """Lengths spread over their logarithm, the least and the most among them; new tokens from none to all, most often all."""
    g = torch.Generator().manual_seed(seed)
    lens = (least * (most / least) ** torch.rand(B, generator=g)).long().clamp(least, most)
    lens[0], lens[-1] = most, least
    n_new = torch.where(torch.rand(B, generator=g) < 0.5, T, torch.randint(0, T + 1, (B,), generator=g))
    n_new[0] = T
    n_new = torch.minimum(n_new, lens)
    return lens.tolist(), n_new.to(torch.int32).cuda()


@pytest.mark.parametrize("B,T,Hq,Hkv,D,dtype,least,most", [
    (16, 64, 32, 8, 64, BF, 3, 6000),      # two tiles of 128 rows, chunks alike
    (16, 64, 32, 8, 128, BF, 70, 9000),
    (4, 64, 32, 8, 128, BF, 64, 6000),     # workgroups for a quarter of the card
    (1, 64, 32, 8, 128, BF, 5000, 5001),
    (64, 40, 32, 8, 80, BF, 1, 3000),      # tiles alone fill the card
    (40, 64, 32, 8, 128, BF, 20, 6100),
    (33, 50, 16, 16, 96, BF, 9, 6000),     # 50 rows of a key head, many heads
    (16, 256, 16, 4, 64, BF, 200, 5000),   # the most nodes, eight tiles
    (64, 8, 32, 8, 128, BF, 1, 6000),      # few rows, split over long caches
    (3, 8, 8, 8, 256, BF, 1, 6000),
    (64, 9, 12, 4, 80, FP, 1, 3000),
    (24, 40, 16, 4, 128, FP, 2, 2500),     # more than 128 rows in 32 bits
])
def test_trees(B, T, Hq, Hkv, D, dtype, least, most):
    lens, n_new = ragged(B, T, least, most, B + T)
    t = inputs(B, T, Hq, Hkv, D, dtype, lens)
    parents = random_tree(B, T, T)
    run(*t, n_new, parents=parents)
    run(*t, n_new, 900, 5, parents)
    run(*t, n_new, parents=parents, max_len=1 << 17)           # what the host knows: right whatever it says


@pytest.mark.parametrize("B,T,Hq,Hkv,D,dtype,least,most,window", [
    (64, 1, 32, 8, 128, BF, 1, 9000, 5500),   # windows that are split
    (64, 1, 32, 8, 128, BF, 1, 9000, 4096),
    (100, 1, 32, 8, 64, BF, 1, 7000, 5000),
    (128, 3, 16, 4, 128, BF, 1, 6000, 5600),
    (16, 5, 32, 8, 80, BF, 1, 9000, 6000),
    (64, 1, 12, 4, 128, FP, 1, 6000, 5000),
    (3, 600, 32, 8, 128, BF, 600, 3000, 700),
])
def test_windows(B, T, Hq, Hkv, D, dtype, least, most, window):
    lens, n_new = ragged(B, T, least, most, B + T)
    t = inputs(B, T, Hq, Hkv, D, dtype, lens)
    run(*t, n_new, window, 0)
    run(*t, n_new, window, 4)


def test_trees_whose_parts_would_be_too_many():
    # chunks that are longer because of what their parts weigh: three of 8192 keys
    B, T = 64, 64
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(64, 400, (B,), generator=g).tolist()
    lens[3], lens[20], lens[41], lens[60] = 24576, 8192, 8193, 17000
    n_new = torch.full((B,), 7, dtype=torch.int32)
    n_new[3], n_new[20], n_new[5] = 64, 40, 0
    run(*inputs(B, T, 32, 8, 128, BF, lens), n_new.cuda(), parents=random_tree(B, T, 3))


def test_holes_in_batches():
    B, T = 24, 64
    lens, n_new = ragged(B, T, 300, 6000, 8)
    q, k, v, table, lens = inputs(B, T, 32, 8, 128, BF, lens)
    drop = torch.rand(table.shape, generator=torch.Generator().manual_seed(9)).cuda() < 0.2
    drop[torch.arange(B), ((lens - 1) // 64).long()] = False                                 # (a row sees itself, or its root, or what is before the tree)
    table = torch.where(drop, torch.tensor([-1, k.shape[0]], device="cuda")[torch.arange(table.shape[1], device="cuda") % 2], table).to(torch.int32)
    n_new = torch.minimum(n_new, (lens - 1) % 64 + 1).to(torch.int32)                         # nodes on the last page, which is there
    run(q, k, v, table, lens, n_new, parents=random_tree(B, T, 4))
    run(q, k, v, table, lens, n_new, 800, 3, random_tree(B, T, 6))


PLANS = [  # B, T, Hq, Hkv, D, dtype, least, most, window of windowed calls (None: trees), max_len
    (16, 64, 32, 8, 128, BF, 70, 9000, None, None), (16, 64, 16, 8, 64, BF, 3, 9000, None, 16384), (40, 64, 32, 8, 128, BF, 20, 6100, None, None),
    (64, 64, 32, 8, 128, BF, 64, 9000, None, 24576), (1, 64, 32, 8, 128, BF, 5000, 5001, None, None), (1, 26, 32, 8, 128, BF, 1999, 2000, None, None),
    (64, 8, 32, 8, 128, BF, 1, 9000, None, None), (64, 9, 12, 4, 80, FP, 1, 3000, None, None), (24, 40, 16, 4, 128, FP, 2, 2500, None, None),
    (64, 1, 32, 8, 128, BF, 1, 9000, 5500, None), (64, 1, 32, 8, 128, BF, 1, 9000, 4096, None), (128, 3, 16, 4, 128, BF, 1, 9000, 5600, None),
    (64, 1, 12, 4, 128, FP, 1, 9000, 5000, None), (3, 600, 32, 8, 128, BF, 600, 3000, 700, None), (2, 300, 4, 4, 64, BF, 300, 9000, 6000, None),
]


@pytest.mark.parametrize("B,T,Hq,Hkv,D,dtype,least,most,window,max_len", PLANS)
def test_no_key_is_lost_or_counted_twice(B, T, Hq, Hkv, D, dtype, least, most, window, max_len):
    # Queries of 0 weigh every key alike, by 1: the denominator is the number of keys, whose logarithm (two units in the last place of 14 in base 2 for every
    # part, and as much for the sum: some 5e-6) tells one of 9000 from none (1e-4).  A value has a 1 at its token's place in the page: counts of every 64th key,
    # divided, rounded once.
    lens, n_new = ragged(B, T, least, most, B + T + 1)
    q, k, v, table, lens = inputs(B, T, Hq, Hkv, D, dtype, lens)
    q.zero_()
    v.zero_()
    place = torch.arange(64, device="cuda")
    v[:, place, :, place % D] = 1.0
    parents = random_tree(B, T, T) if window is None else None
    for w, sinks in ((window or ALL, 0), (window or 900, 5)):
        kw = dict(max_len=max_len, n_new=n_new, want_lse=True, sinks=sinks)
        out, lse = (tsd.window_attn_static(q, k, v, table, lens, w, **kw) if parents is None else
                    tsd.tree_attn_static(q, k, v, table, lens, parents.cuda(), window=None if w == ALL else w, **kw))
        for b, (length, n) in enumerate(zip(lens.tolist(), n_new.tolist())):
            if not n:
                continue
            sees = sight(length, n, w, sinks, None if parents is None else parents[b]).cuda()
            total = sees.sum(1).double()
            assert float((lse[b, :n].double() - torch.log(total)[:, None]).abs().max()) <= 1e-5, (b, w)
            each = torch.nn.functional.pad(sees.double(), (0, -sees.shape[1] % 64)).view(n, -1, 64).sum(1)
            want = torch.zeros(n, D, dtype=torch.float64, device="cuda").index_add_(1, place % D, each) / total[:, None]
            assert bool(((out[b, :n].double() - want[:, None]).abs() <= (HALF[dtype] + 1e-5) * want[:, None]).all()), (b, w)
