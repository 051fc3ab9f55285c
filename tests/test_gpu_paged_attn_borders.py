"""No key is lost or counted twice where a step, a tile or a chunk of keys ends: every row has one key that takes half of its weight, and those keys go
over all multiples of 32 and their neighbours, and over the border of what a row sees."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import F32, HALF

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def check(dtype, B, T, Hq, Hkv, D, n, heavy, seed=0, page=16):
    """heavy: [B, Hkv, rows a key head], the key that row t * G + g of a key head weighs as much as all others together."""
    G, cols = Hq // Hkv, -(-n // page)
    rows = T * G
    g = torch.Generator().manual_seed(seed)
    table = torch.randperm(B * cols, generator=g).to(torch.int32).view(B, cols)
    # scores: ln(n) for the heavy keys, 0 for all others; a row's direction is a dim (rows that share one share their heavy keys)
    dims = torch.arange(rows) % D
    k, q = torch.zeros(B, n, Hkv, D, dtype=torch.float64), torch.zeros(B, T, Hq, D, dtype=torch.float64)
    b, h, r = (x.flatten() for x in torch.meshgrid(torch.arange(B), torch.arange(Hkv), torch.arange(rows), indexing="ij"))
    q[b, r // G, h * G + r % G, dims[r]] = 4.0
    k[b, heavy[b, h, r], h, dims[r]] = math.log(n) * math.sqrt(D) / 4
    v = torch.randn(B, n, Hkv, D, generator=g, dtype=torch.float64)
    v[b, heavy[b, h, r], h] *= 8
    q, k, v = q.to(dtype).double(), k.to(dtype).double(), v.to(dtype).double()
    pools = []
    for x in (k, v):
        pool = torch.zeros(B * cols * page, Hkv, D, dtype=torch.float64)
        slots = torch.arange(n)
        for s in range(B):
            pool[table[s, slots // page].long() * page + slots % page] = x[s]
        pools.append(pool.view(-1, page, Hkv, D).to(dtype).cuda())
    lens = torch.full((B,), n, dtype=torch.int32).cuda()
    got, lse = tsd.paged_attn_static(q.to(dtype).cuda(), *pools, table.cuda(), lens, want_lse=True)
    k, v = k.repeat_interleave(G, 2), v.repeat_interleave(G, 2)
    s = torch.einsum("bthd,bnhd->bthn", q, k) / math.sqrt(D)
    s.masked_fill_((torch.arange(n)[None] > (n - T + torch.arange(T))[:, None])[None, :, None], -math.inf)
    w = torch.softmax(s, -1)
    want, mass = torch.einsum("bthn,bnhd->bthd", w, v), torch.einsum("bthn,bnhd->bthd", w, v.abs())
    # a score has one product that is not 0: its rounding, the factor's and the difference's; weights and their sums in the values' type at worst; n sums
    half = HALF[dtype]
    rel = 8 * F32 * 1.5 * math.log(n) + (n + 44) * F32 + (half if dtype == BF else 0.0)
    off = (got.double().cpu() - want).abs()
    assert bool((off <= 1.05 * rel * (mass + want.abs()) + half * want.abs()).all())
    assert bool(((lse.double().cpu() - torch.logsumexp(s, -1)).abs() <= rel + 4 * F32 * 10).all())
    return w


SIZES = [
    (1, 1, 16, 1, 64, 61), (2, 2, 4, 2, 64, 1000),                      # whole, joined in the launch
    (1, 5, 32, 8, 128, 4099), (3, 1, 8, 1, 64, 2500), (2, 3, 2, 2, 256, 1300), (1, 9, 4, 1, 80, 2000),      # a second launch; wide and odd heads
    (1, 70, 2, 2, 64, 500), (2, 130, 1, 1, 128, 500), (2, 130, 1, 1, 128, 250),      # many rows: short chunks, whole
    (1, 80, 2, 2, 128, 3100), (2, 65, 4, 1, 96, 1700), (1, 200, 2, 1, 64, 4099),
]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,n", SIZES)
def test_multiples_of_a_step(dtype, B, T, Hq, Hkv, D, n):
    rows = T * (Hq // Hkv)
    # keys that every row sees
    at = sorted({j for m in range(0, n + 32, 32) for j in (m - 1, m, m + 1) if 0 <= j <= n - T} | {0, n - T})
    each = B * Hkv * rows
    for first in range(0, len(at), each):
        heavy = torch.tensor([at[(first + i) % len(at)] for i in range(each)]).view(B, Hkv, rows)
        w = check(dtype, B, T, Hq, Hkv, D, n, heavy, seed=first)
        if rows <= D:
            assert 0.4 < float(w.amax(-1).min()) and float(w.amax(-1).max()) < 0.6


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,n", [s for s in SIZES if s[1] > 1])
@pytest.mark.parametrize("ahead", [0, 1])
def test_the_last_key_that_a_row_sees_and_the_next(dtype, B, T, Hq, Hkv, D, n, ahead):
    G = Hq // Hkv
    own = n - T + torch.arange(T * G) // G
    check(dtype, B, T, Hq, Hkv, D, n, (own + ahead).clamp(max=n - 1).expand(B, Hkv, -1), seed=ahead)
