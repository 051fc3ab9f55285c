"""token_logprobs_static against its definition in 64 bits (tests/tree_ref.py), within bounds that count roundings."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from tree_ref import check_scores, scores

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32
LOWEST = {BF: torch.finfo(BF).min, FP: torch.finfo(FP).min}


def inputs(B, T, V, dtype, seed=0, spread=3.0, wide=True):
    g = torch.Generator().manual_seed(seed)
    logits = (spread * torch.randn(B, T, V, generator=g)).to(dtype).cuda()
    return logits, torch.randint(0, V, (B, T), generator=g).to(torch.int64 if wide else torch.int32).cuda()


def run(logits, tokens, top=0, temperature=1.0, n_new=None):
    got = tsd.token_logprobs_static(logits, tokens, top=top, temperature=temperature, n_new=n_new)
    check_scores(got, *scores(logits, tokens, top, temperature, n_new), tokens=tokens is not None)
    return got


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("top", [0, 1, 5, 32])
@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (1, 1, 2), (2, 3, 31), (1, 2, 64), (3, 1, 255), (2, 2, 1000), (1, 1, 1024), (1, 3, 1025), (2, 1, 4099), (1, 1, 32000),
                                   (2, 2, 50257), (1, 1, 65537), (1, 1, 131072), (1, 1, 300001), (200, 1, 70000)])
def test_sizes(dtype, top, B, T, V):
    run(*inputs(B, T, V, dtype), top)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B,T,V", [(600, 1, 50), (70, 8, 3001), (130, 4, 20000), (513, 1, 17000)])
@pytest.mark.parametrize("top", [0, 7])
def test_many_rows(dtype, B, T, V, top):
    # a workgroup a row
    run(*inputs(B, T, V, dtype, wide=False), top)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_very_many_rows(dtype):
    # the same rows over and over
    logits, tokens = inputs(5, 100, 37, dtype)
    some = run(logits, tokens, 3)
    all_of = tsd.token_logprobs_static(logits.repeat(110, 10, 1), tokens.repeat(110, 10), top=3)
    for name, x in some.items():
        assert torch.equal(all_of[name], x.repeat(110, 10, *[1] * (x.dim() - 2))), name


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("temperature", [0.05, 0.7, 1.3, 100.0])
def test_temperatures(dtype, temperature):
    run(*inputs(2, 3, 5000, dtype), 4, temperature)
    run(*inputs(300, 2, 500, dtype), 4, temperature)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B", [2, 520])
@pytest.mark.parametrize("V", [100, 5000, 40000, 100000])
def test_ties_go_to_the_lowest_index(dtype, B, V):
    # every logit the same; a few values; ties at the border of what is asked for
    logits, tokens = inputs(B, 1, V, dtype)
    run(torch.zeros_like(logits), tokens, 32)
    run(torch.round(logits[:2] / 3), tokens[:2], 20)
    x = torch.full_like(logits, -2.0)
    x[:, :, V // 3] = 5.0
    x[:, :, V - 2:] = 1.0
    run(x, tokens, 9)
    signed = torch.zeros_like(logits)
    signed[..., ::2] = -0.0                                   # zeros are the same whatever their sign
    run(signed, tokens, 5)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B", [2, 520])
@pytest.mark.parametrize("left", [0, 1, 3, 40])
def test_masked_logits(dtype, B, left):
    # all but a few tokens masked, by -inf and by the type's lowest value
    V = 9000 if B > 2 else 100000
    logits, tokens = inputs(B, 1, V, dtype)
    some = torch.randperm(V, generator=torch.Generator().manual_seed(2))[:left]
    for mask in (-math.inf, LOWEST[dtype], -1e9):
        x = torch.full_like(logits, mask)
        x[..., some] = logits[..., some]
        tokens[0, 0] = int(some[0]) if left else 5
        run(x, tokens, 10)
        run(x, tokens, 0, 0.5)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("B", [1, 600])
def test_orders_that_are_hard_for_bounds(dtype, B):
    # logits that rise, that fall, whose largest lie in one lane's elements, or in one wavefront's only
    V = 20000 if B > 1 else 100000
    up = torch.linspace(-8, 8, V).expand(B, 1, V).to(dtype).cuda().contiguous()
    tokens = torch.full((B, 1), V // 2, dtype=torch.int64).cuda()
    run(up, tokens, 32)
    run(up.flip(-1).contiguous(), tokens, 32)
    x, _ = inputs(B, 1, V, dtype, spread=1.0)
    step = 256 * (8 if dtype == BF else 4)
    x[..., 3::step] += 30                                     # the same lane's, once a load
    run(x, tokens, 20)
    lane = torch.arange(V) % step // (step // 256)
    y = torch.full_like(x, -math.inf)
    y[..., lane < 64] = x[..., lane < 64]                     # nothing in three of the four wavefronts: thousands reach what bound there is
    run(y, tokens, 20)
    run(torch.where(torch.isfinite(y), y, LOWEST[dtype]), tokens, 20)


def test_values_that_are_none():
    logits, tokens = inputs(4, 2, 3000, FP)
    logits[0, 0, 7], logits[1, 0, 9], logits[1, 1] = math.nan, math.inf, -math.inf
    tokens[0, 1], tokens[2, 0], tokens[2, 1], tokens[3, 0] = -1, 3000, -100, 2 ** 40
    logits[3, 1, 100] = -math.inf
    tokens[3, 1] = 100
    got = tsd.token_logprobs_static(logits, tokens, top=6)
    clean = [(0, 1), (2, 0), (2, 1), (3, 0), (3, 1), (1, 1)]
    want, tol = scores(logits, tokens, 6)
    pick = lambda x: torch.stack([x[c] for c in clean])[:, None]
    import numpy as np
    npick = lambda x: np.stack([x[c] for c in clean])[:, None]
    check_scores({k: pick(v) for k, v in got.items()}, [npick(x) for x in want], [npick(x) for x in tol])
    for c in ((0, 0), (1, 0)):
        assert bool(got["logprobs"][c].isnan()) and bool(got["entropy"][c].isnan()) and bool(got["top_logprobs"][c].isnan().all())
    # NaN is never among the likeliest, an infinite logit is the first
    finite = torch.where(logits[0, 0].isnan(), -math.inf, logits[0, 0])
    assert got["top_ids"][0, 0].tolist() == finite.cpu().sort(descending=True, stable=True).indices[:6].tolist()
    assert int(got["top_ids"][1, 0, 0]) == 9
    assert got["top_ids"][1, 1].tolist() == [-1] * 6 and float(got["entropy"][1, 1]) == 0.0 and float(got["logprobs"][1, 1]) == -math.inf


@pytest.mark.parametrize("dtype", [BF, FP])
def test_the_largest_and_smallest_logits(dtype):
    V, big = 2000, torch.finfo(dtype).max
    logits, tokens = inputs(3, 1, V, dtype)
    logits[0, 0, :50], logits[0, 0, 50:] = big, -big
    logits[1] = -big
    logits[2, 0, 3] = big
    tokens[0, 0], tokens[1, 0], tokens[2, 0] = 7, 0, 3
    got = tsd.token_logprobs_static(logits, tokens, top=3)
    assert got["logprobs"].tolist() == [[pytest.approx(-math.log(50), rel=1e-6)], [pytest.approx(-math.log(V), rel=1e-6)], [0.0]]
    assert got["entropy"].tolist() == [[pytest.approx(math.log(50), rel=1e-6)], [pytest.approx(math.log(V), rel=1e-6)], [0.0]]
    assert got["top_ids"].tolist()[:2] == [[[0, 1, 2]], [[0, 1, 2]]] and int(got["top_ids"][2, 0, 0]) == 3


@pytest.mark.parametrize("B,T,V", [(3, 5, 3000), (200, 4, 700)])
def test_ragged_rows(B, T, V):
    logits, tokens = inputs(B, T, V, BF)
    n_new = (torch.arange(B) * 3 % (T + 3) - 1).to(torch.int32).cuda()       # below 0 and above T: clamped
    for b in range(B):
        logits[b, max(int(n_new[b]), 0):] = math.nan                         # rows behind are not read
    got = run(logits, tokens, 4, 1.0, n_new)
    assert bool(torch.isfinite(got["logprobs"]).all())
    run(logits, None, 4, 1.0, n_new)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_strides(dtype):
    wide, tokens = inputs(3, 4, 1111, dtype)
    run(wide[:, :, 1:1002], tokens % 1001, 3)                                # rows that start anywhere
    run(wide.transpose(0, 1), tokens.t().contiguous(), 3)
    run(wide[:, :1].expand(3, 4, 1111), tokens, 3)
    run(wide[:, ::2], tokens[:, ::2].contiguous(), 3)


def test_repeated_calls_give_the_same_bits():
    for B, V in ((1, 100000), (4, 5000), (700, 3000)):
        logits, tokens = inputs(B, 1, V, BF)
        first = tsd.token_logprobs_static(logits, tokens, top=20)
        for _ in range(20):
            again = tsd.token_logprobs_static(logits, tokens, top=20)
            assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("B,V", [(1, 100000), (600, 3000)])
def test_streams_and_replayed_graphs(B, V):
    logits, tokens = inputs(B, 1, V, BF)
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                got = tsd.token_logprobs_static(logits, tokens, top=8)
            graphs.append((g, got))
    torch.cuda.synchronize()
    for step in range(5):
        logits.normal_().mul_(1.0 + step)
        torch.cuda.synchronize()
        want = tsd.token_logprobs_static(logits, tokens, top=8)
        for s, (g, got) in zip(streams, graphs):
            for x in got.values():
                x.zero_()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for _, got in graphs:
            assert all(torch.equal(want[k], got[k]) for k in want)


def test_offsets_beyond_32_bits():
    V, T = 1 << 20, 4200                                       # elements past 2^32, 8.8 GB
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs some 12 GB of device memory")
    logits = torch.empty(1, T, V, dtype=BF, device="cuda")
    some, tokens = inputs(1, 3, V, BF)
    rows = [0, 4097, T - 1]
    logits[:, rows] = some
    n = torch.zeros(1, T, dtype=torch.int64, device="cuda")
    n[:, rows] = tokens
    logits[:, [r for r in range(T) if r not in rows]] = 0.0
    got = tsd.token_logprobs_static(logits, n, top=3)
    check_scores({k: v[:, rows] for k, v in got.items()}, *scores(some, tokens, 3))
