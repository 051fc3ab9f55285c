"""rope_append_static against its definition in 64 bits (tests/round_ref.py)."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import paged, rotated

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def case(B, T, Hq, Hkv, D, page, dtype, cols, seed=0, order="token"):
    g = torch.Generator().manual_seed(seed)
    new = lambda h: torch.randn(B, T, h, D, generator=g).to(dtype).cuda()
    return new(Hq), new(Hkv), new(Hkv), *paged(B, cols, page, Hkv, D, dtype, seed, order, spare=2, fill=3.0)


def check(q, k, v, k_pool, v_pool, table, base, freq, positions=None, n_new=None, interleaved=False, amplitude=1.0, out=None):
    B, T = q.shape[:2]
    page, n_pages = k_pool.shape[1], k_pool.shape[0]
    slots = base.cpu()[:, None] + torch.arange(T)[None]
    pos = slots if positions is None else positions.cpu()
    yq, tq = rotated(q, pos, freq, interleaved, amplitude)
    yk, tk = rotated(k, pos, freq, interleaved, amplitude)
    there = torch.ones(B, T, dtype=torch.bool) if n_new is None else torch.arange(T)[None] < n_new.cpu().clamp(0, T)[:, None]
    want_k, want_v, tol_k = k_pool.double().cpu(), v_pool.double().cpu(), torch.zeros(k_pool.shape, dtype=torch.float64)
    for b in range(B):
        for t in range(T):
            s = int(slots[b, t])
            if not there[b, t] or s < 0 or s // page >= table.shape[1] or not 0 <= int(table[b, s // page]) < n_pages:
                continue
            at = int(table[b, s // page]), s % page
            want_k[at], tol_k[at], want_v[at] = yk[b, t], tk[b, t], v[b, t].double().cpu()
    before = None if out is None or out is q else out.clone()
    got = tsd.rope_append_static(q, k, v, k_pool, v_pool, table, base, freq, positions, n_new, interleaved, amplitude, out)
    off = (got.double().cpu() - yq).abs()
    assert bool((off[there] <= tq[there]).all()), float((off / tq.clamp(min=1e-30))[there].max())
    if before is not None:
        assert torch.equal(got.cpu()[~there], before.cpu()[~there])
    off = (k_pool.double().cpu() - want_k).abs()
    assert bool((off <= tol_k).all()), float(off.max())         # what nobody writes keeps its bits
    assert torch.equal(v_pool.double().cpu(), want_v)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,T,Hq,Hkv,D,R,page", [
    (1, 1, 1, 1, 64, 64, 16), (3, 5, 6, 2, 128, 128, 16), (2, 3, 4, 4, 80, 32, 8), (2, 2, 3, 1, 64, 2, 1), (2, 7, 5, 5, 96, 20, 64),
    (1, 3, 2, 1, 256, 256, 32), (2, 2, 3, 3, 8, 8, 16), (2, 2, 2, 1, 16, 16, 4), (300, 2, 2, 1, 64, 48, 16), (1, 2, 40, 8, 128, 64, 16),
])
def test_sizes(dtype, interleaved, B, T, Hq, Hkv, D, R, page):
    q, k, v, kp, vp, table = case(B, T, Hq, Hkv, D, page, dtype, cols=-(-(40 + T) // page))
    base = torch.arange(B, dtype=torch.int32).cuda() % 41
    freq, amplitude = tsd.rope_frequencies(R)
    check(q, k, v, kp, vp, table, base, freq, interleaved=interleaved, amplitude=amplitude)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("scaling", [None, "linear", "base", "blend"])
def test_far_positions_and_scalings(dtype, scaling):
    q, k, v, kp, vp, table = case(4, 3, 4, 2, 64, 16, dtype, cols=2)
    base = torch.tensor([0, 5, 16, 29], dtype=torch.int32).cuda()
    freq, amplitude = tsd.rope_frequencies(64, scaling=scaling, factor=4.0, original_len=4096)
    positions = torch.tensor([[0, 1, 2], [100000, 5, 99999], [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 24 + 1], [7, 7, -3]], dtype=torch.int32).cuda()
    check(q, k, v, kp, vp, table, base, freq, positions, amplitude=amplitude)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_ragged_in_place_and_slots_without_a_page(dtype):
    q, k, v, kp, vp, table = case(5, 4, 4, 2, 64, 16, dtype, cols=3, order="head")
    freq, _ = tsd.rope_frequencies(64)
    n_new = torch.tensor([0, 4, 2, 99, -1], dtype=torch.int32).cuda()
    base = torch.tensor([3, 14, 46, 0, 1], dtype=torch.int32).cuda()
    out = torch.full_like(q, 7.0)
    check(q, k, v, kp, vp, table, base, freq, n_new=n_new, out=out)
    table[1, 0], table[3, 0] = -1, kp.shape[0]                # holes: the queries turn all the same
    base = torch.tensor([3, 14, 47, 0, -2], dtype=torch.int32).cuda()
    check(q, k, v, kp, vp, table, base, freq, out=out)
    kept = q.clone()
    got = tsd.rope_append_static(q, k, v, kp, vp, table, base, freq, n_new=n_new, out=q)
    want = tsd.rope_append_static(kept, k, v, kp, vp, table, base, freq, n_new=n_new, out=kept.clone())
    assert got.data_ptr() == q.data_ptr() and torch.equal(q, want)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_strides(dtype):
    B, T, Hq, Hkv, D = 2, 3, 4, 2, 64
    g = torch.Generator().manual_seed(3)
    fused = torch.randn(B, T, Hq + 2 * Hkv, D, generator=g).to(dtype).cuda()
    q, k, v = fused.split([Hq, Hkv, Hkv], 2)
    both = torch.full((9, 2, Hkv, 16, D), 3.0).to(dtype).cuda()
    kp, vp = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    table = torch.randperm(9, generator=g)[:6].to(torch.int32).view(2, 3).cuda()[:, 1:]
    out = torch.full((B, T, Hq, 2 * D), 7.0, dtype=dtype).cuda()
    freq, _ = tsd.rope_frequencies(D)
    base = torch.tensor([0, 15], dtype=torch.int32).cuda()
    check(q, k, v, kp, vp, table, base, freq, out=out[..., :D])
    assert bool((out[..., D:] == 7.0).all())
    check(q, k[:, :, :1].expand(B, T, Hkv, D), v, kp, vp, table, base, freq)       # one key for all heads


def test_offsets_beyond_32_bits():
    page, Hkv, D = 64, 8, 128
    n = (1 << 32) // (page * Hkv * D) + 40
    if torch.cuda.mem_get_info()[0] < 3 * n * page * Hkv * D * 2:
        pytest.skip("needs some 25 GB of device memory")
    kp, vp = (torch.empty(n, page, Hkv, D, dtype=BF, device="cuda") for _ in range(2))
    q, k, v, skp, svp, _ = case(1, 3, 8, Hkv, D, page, BF, cols=1)
    freq, _ = tsd.rope_frequencies(D)
    base = torch.tensor([63], dtype=torch.int32).cuda()
    pages = [n - 1, n // 2 + 7]
    tsd.rope_append_static(q, k, v, kp, vp, torch.tensor([pages], dtype=torch.int32).cuda(), base, freq)
    tsd.rope_append_static(q, k, v, skp, svp, torch.tensor([[0, 1]], dtype=torch.int32).cuda(), base, freq)
    for big, small in ((kp, skp), (vp, svp)):
        assert torch.equal(big[n - 1, 63], small[0, 63]) and torch.equal(big[n // 2 + 7, :2], small[1, :2])


def test_replayed_graph():
    q, k, v, kp, vp, table = case(2, 3, 4, 2, 64, 16, BF, cols=4)
    freq, _ = tsd.rope_frequencies(64)
    base, out = torch.tensor([0, 7], dtype=torch.int32).cuda(), torch.zeros_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            tsd.rope_append_static(q, k, v, kp, vp, table, base, freq, out=out)
    for step in range(4):
        q.normal_()
        base += step
        g.replay()
        torch.cuda.synchronize()
        other = [kp.clone(), vp.clone()]
        want = tsd.rope_append_static(q, k, v, *other, table, base, freq)
        assert torch.equal(out, want) and torch.equal(kp, other[0]) and torch.equal(vp, other[1])
