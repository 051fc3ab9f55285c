"""How the bf16 attention kernels weigh: a weight's rounding moves a row only by its share of the distance between its value and the result, and the
heaviest weight, which is 1, not at all.  Few rows a key head and many run in different kernels; both are held to this.

Scores are exact here (queries and keys are multiples of 1/4 and 1/8, so that their products add up without rounding), which leaves the weights' and
the result's rounding to bf16 as all that is large."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import F32, HALF, paged

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def inputs(T, Hq, Hkv, D, n, deviation, seed=0, page=16):
    g = torch.Generator().manual_seed(seed)
    k, v, table = paged(1, -(-n // page), page, Hkv, D, BF, seed)
    k = (k.float() * 8).round().clamp(-32, 32).div(8).to(BF)
    q = (deviation * torch.randn(1, T, Hq, D, generator=g) * 4).round().clamp(-128, 128).div(4).to(BF).cuda()
    return q, k, v, table, torch.tensor([n], dtype=torch.int32).cuda()


def exact(q, k, v, table, lens):
    """out, logarithm of the denominator, how far off each may be: float64 [T, Hq, D] and [T, Hq]."""
    n, (T, Hq, D), G = int(lens[0]), q.shape[1:], q.shape[2] // k.shape[2]
    at = table[0].long()
    k, v = (x[at].flatten(0, 1)[:n].double().cpu().repeat_interleave(G, 1) for x in (k, v))      # [n, Hq, D]
    s = torch.einsum("thd,nhd->thn", q[0].double().cpu(), k) / math.sqrt(D)
    s.masked_fill_(torch.arange(n)[None, None] > (n - T + torch.arange(T))[:, None, None], -math.inf)
    w = torch.softmax(s, -1)
    out, lse = torch.einsum("thn,nhd->thd", w, v), torch.logsumexp(s, -1)
    # Scores: the factor, in base 2 from two roundings, one product and one difference: 4 roundings of the largest score, for a weight and for the
    # maximum each; exp2, 4; sums over n keys, n roundings.
    rel = (8 * F32 * 1.45 * s.masked_fill(s == -math.inf, 0).abs().amax(-1) + (n + 44) * F32)[..., None]
    far = (w[:, :, None] * (v.permute(1, 2, 0)[None] - out[..., None]).abs())                     # [T, Hq, D, n]: share times distance
    top = w.argmax(-1)
    far = far.sum(-1) - far.gather(3, top[..., None, None].expand(*far.shape[:3], 1))[..., 0]
    half = HALF[BF]
    mass = torch.einsum("thn,nhd->thd", w, v.abs())
    tol = half / (1 - half) * far + rel * (mass + out.abs())
    return out, lse, tol + half * (out.abs() + tol), rel[..., 0], half * (1 - w.amax(-1))


SIZES = [(3, 8, 2, 128, 700), (1, 4, 4, 64, 90), (20, 2, 2, 80, 2000), (65, 2, 2, 128, 700), (200, 2, 2, 64, 300), (130, 1, 1, 96, 2500), (80, 2, 1, 128, 1500)]


@pytest.mark.parametrize("T,Hq,Hkv,D,n", SIZES)
@pytest.mark.parametrize("deviation", [1.5, 4.0, 8.0])
def test_the_heaviest_weight_is_exact_and_others_move_a_row_by_their_distance(T, Hq, Hkv, D, n, deviation):
    q, k, v, table, lens = inputs(T, Hq, Hkv, D, n, deviation)
    out, lse, tol, rel, of_lse = exact(q, k, v, table, lens)
    got, got_lse = tsd.paged_attn_static(q, k, v, table, lens, want_lse=True)
    off = (got[0].double().cpu() - out).abs()
    assert bool((off <= tol).all()), float((off / tol).max())
    # (a sum of rounded weights at worst)
    off = (got_lse[0].double().cpu() - lse).abs()
    assert bool((off <= rel + of_lse * (1 + HALF[BF]) + 4 * F32 * lse.abs()).all())


@pytest.mark.parametrize("T,Hq,Hkv,D,n", SIZES)
@pytest.mark.parametrize("deviation", [0.0, 1.5, 4.0, 8.0])
def test_weights_add_up_to_one(T, Hq, Hkv, D, n, deviation):
    # values of 1: both sums are of the same weights, and differ by n + 44 roundings of 2^-24 each way at most, far less than bf16 shows
    q, k, v, table, lens = inputs(T, Hq, Hkv, D, n, deviation, seed=3)
    v.fill_(1.0)
    assert 2 * (n + 44) * F32 < HALF[BF] / 2
    assert bool((tsd.paged_attn_static(q, k, v, table, lens) == 1.0).all())
