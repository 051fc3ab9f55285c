"""verify_tokens_static against its definition in 64 bits (tests/round_ref.py): counts and tokens are equal."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from round_ref import verified

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def inputs(B, K, V, dtype, seed=0, noise=0.5, token=torch.int64):
    g = torch.Generator().manual_seed(seed)
    logits = 2.0 * torch.randn(B, K + 1, V, generator=g)
    p = torch.softmax(logits, -1).to(dtype)
    q = torch.softmax(logits[:, :K] + noise * torch.randn(B, K, V, generator=g), -1).to(dtype)
    draft = torch.multinomial(q.float().reshape(-1, V), 1, generator=g).view(B, K).to(token)
    return [x.cuda() for x in (draft, q, p, torch.rand(B, K + 1, generator=g))]


def check(draft, q, p, u, n_draft=None):
    got = tsd.verify_tokens_static(draft, q, p, u, n_draft=n_draft)
    n, tokens = verified(draft, q, p, u, n_draft)
    assert got["n_acc"].dtype == torch.int32 and got["tokens"].dtype == draft.dtype
    assert got["n_acc"].tolist() == n
    assert got["tokens"].tolist() == tokens
    return n, tokens


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (2, 3, 2), (5, 4, 7), (3, 16, 63), (4, 2, 1023), (4, 2, 1024), (4, 5, 1025), (7, 4, 5001), (2, 3, 32000),
                                   (3, 4, 50257), (1, 2, 262147), (700, 3, 33)])
def test_sizes(dtype, B, K, V):
    n, _ = check(*inputs(B, K, V, dtype))
    check(*inputs(B, K, V, dtype, seed=1, token=torch.int32))
    if B > 4 and V > 2:
        assert 0 < sum(n) < B * K


@pytest.mark.parametrize("dtype", [FP, BF])
def test_ragged_drafts_and_certain_ones(dtype):
    draft, q, p, u = inputs(6, 4, 300, dtype, noise=0.1)
    n_draft = torch.tensor([0, 1, 2, 4, 99, -1], dtype=torch.int32).cuda()
    check(draft, q, p, u, n_draft)
    draft = p[:, :4].argmax(-1)
    u = u * 0.05
    check(draft, None, p, u, n_draft)
    check(draft, None, p, u)
    one = torch.zeros_like(p)
    one.scatter_(2, p.argmax(-1, keepdim=True), 1.0)          # greedy decoding: one token has it all
    draft[:, 2] = (draft[:, 2] + 1) % 300
    n, tokens = check(draft, None, one, torch.rand(6, 5).cuda())
    assert n == [2] * 6 and [t[2] for t in tokens] == one[:, 2].argmax(-1).tolist()


def test_borders():
    # dyadic probabilities: sums are exact, draws on a border go to the token behind it
    V = 4096
    p = torch.full((1, 2, V), 1.0 / V).cuda()
    q = p[:, :1].clone()
    draft = torch.tensor([[5]]).cuda()
    for x in (0.0, 0.25, 0.5, 1023 / V, 1024 / V, (V - 1) / V, 1 - 2 ** -24):
        check(draft, q, p, torch.tensor([[0.5, x]]).cuda())
    # equal probabilities: every draft passes for u < 1; a draw of u = 0 where p = 0 does not
    assert check(draft, q, p, torch.tensor([[1 - 2 ** -24, 0.5]]).cuda())[0] == [1]
    p[0, 0, 5] = 0
    assert check(draft, q, p, torch.tensor([[0.0, 0.5]]).cuda())[0] == [0]
    # zero weights are never drawn, at neither end
    p = torch.zeros(1, 2, V).cuda()
    p[0, :, 1500] = 0.25
    p[0, :, 1501] = 0.25
    for x in (0.0, 0.499, 0.5, 1 - 2 ** -24, 1.0, 2.0, -1.0, math.nan):
        check(draft, q, p, torch.tensor([[0.9, x]]).cuda())


@pytest.mark.parametrize("V", [50, 5000])
def test_values_that_are_no_probabilities(V):
    draft, q, p, u = inputs(8, 3, V, FP, seed=3)
    p[0, :, ::3] = math.nan
    q[1, :, 1::2] = math.nan
    p[2] = 0.0                                            # nothing to draw
    p[3, :, 7] = math.inf
    q[4], p[4] = 1.0, 0.5                                 # nothing left of p over q: by p
    p[5] = -p[5]
    draft[6, 1] = V                                       # no token
    draft[7, 0] = -1
    u[4, 0] = 0.9
    n, tokens = check(draft, q, p, u)
    assert tokens[2][0] == -1 and n[2] == 0
    check(draft, None, p, u)


def test_strides_and_odd_starts():
    draft, q, p, u = inputs(4, 3, 777, BF)
    wide_p, wide_q = torch.zeros(4, 4, 801, dtype=BF).cuda(), torch.zeros(3, 4, 779, dtype=BF).cuda()
    wide_p[:, :, 3:780], wide_q[:, :, 1:778] = p, q.transpose(0, 1)
    check(draft, wide_q.transpose(0, 1)[..., 1:778], wide_p[..., 3:780], u)
    check(draft, q[:, :1].expand(4, 3, 777), p[:1].expand(4, 4, 777), u)
    draft, q, p, u = inputs(4, 3, 777, FP)
    flat = torch.zeros(p.numel() + 1).cuda()
    flat[1:] = p.flatten()
    check(draft, q, flat[1:].view_as(p), u)


def test_sums_of_many_small_terms():
    # a sum in 32 bits would lose every term behind the first
    V = 200000
    p = torch.full((2, 2, V), 2.0 ** -26).cuda()
    p[:, :, 0] = 1.0
    q, draft = torch.zeros(2, 1, V).cuda(), torch.tensor([[0], [0]]).cuda()
    u = torch.tensor([[0.5, 1 - 2 ** -24], [0.5, 0.9985]]).cuda()
    check(draft, q, p, u)


def test_distribution():
    """What comes out first is distributed as the target says, whatever the draft proposes: 20000 sequences, a chi-square of 7 degrees."""
    B, V = 20000, 8
    g = torch.Generator().manual_seed(11)
    p1 = torch.tensor([0.3, 0.2, 0.15, 0.1, 0.1, 0.08, 0.05, 0.02])
    q1 = torch.tensor([0.1, 0.1, 0.3, 0.05, 0.2, 0.05, 0.15, 0.05])
    draft = torch.multinomial(q1, B, replacement=True, generator=g).view(B, 1).cuda()
    got = tsd.verify_tokens_static(draft, q1.expand(B, 1, V).cuda(), p1.expand(B, 2, V).cuda(), torch.rand(B, 2, generator=g).cuda())
    counts = torch.bincount(got["tokens"][:, 0].cpu(), minlength=V).double()
    chi = float(((counts - B * p1.double()) ** 2 / (B * p1.double())).sum())
    assert chi < 24.3                                     # the 0.999 quantile; the seed is fixed
    share = float(got["n_acc"].double().mean())
    want = float(torch.minimum(p1, q1).sum())
    assert abs(share - want) < 4 * math.sqrt(want * (1 - want) / B)


def test_replayed_graph_and_streams():
    draft, q, p, u = inputs(4, 3, 3000, FP)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got = tsd.verify_tokens_static(draft, q, p, u)
    for seed in range(3):
        for to, x in zip((draft, q, p, u), inputs(4, 3, 3000, FP, seed=seed)):
            to.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        n, tokens = verified(draft, q, p, u)
        assert got["n_acc"].tolist() == n and got["tokens"].tolist() == tokens
        check(draft, q, p, u)


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("B,V", [(1, 40000), (3, 131072), (130, 33000)])
def test_rows_shared_by_workgroups(dtype, B, V):
    # the last workgroup of a row draws: again in the same memory, replayed, and with nothing left of p over q
    draft, q, p, u = inputs(B, 2, V, dtype)
    check(draft, q, p, u)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got = [tsd.verify_tokens_static(draft, q, p, u), tsd.verify_tokens_static(draft, None, p, u)]
    torch.cuda.synchronize()
    for step in range(5):
        u.uniform_()
        if step == 3:
            p[0], q[0] = 2.0 ** -18, 2.0 ** -17
        g.replay()
        torch.cuda.synchronize()
        for x, by in zip(got, (q, None)):
            n, tokens = verified(draft, by, p, u)
            assert x["n_acc"].tolist() == n and x["tokens"].tolist() == tokens
        check(draft, q, p, u)
