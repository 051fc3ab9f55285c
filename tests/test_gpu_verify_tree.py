"""verify_tree_static against its definition (tests/tree_ref.py): whole numbers, equal."""
import math

import pytest
import torch

import paper_2511_18191_amd as tsd
from tree_ref import random_tree, walked

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32


def inputs(B, N, V, dtype=FP, seed=0, wide=False, sharp=4.0):
    """Trees whose nodes are likely tokens, siblings different where the vocabulary has enough."""
    g = torch.Generator().manual_seed(seed)
    p = torch.softmax(sharp * torch.randn(B, N, V, generator=g), -1)
    parents = random_tree(B, N, seed + 1)
    likely = p.topk(min(4, V), -1).indices
    tokens = torch.zeros(B, N, dtype=torch.long)
    for b in range(B):
        born = [0] * N
        for n in range(1, N):
            up = int(parents[b, n])
            tokens[b, n] = likely[b, up, born[up] % likely.shape[2]]
            born[up] += 1
    u = torch.rand(B, N, generator=g)
    return tokens.to(torch.int64 if wide else torch.int32).cuda(), parents.cuda(), p.to(dtype).cuda(), u.cuda()


def run(tokens, parents, p=None, u=None, choices=None, n_new=None):
    got = tsd.verify_tree_static(tokens, parents, p=p, uniforms=u, choices=choices, n_new=n_new)
    n_acc, out, path = walked(tokens, parents, p, u, choices, n_new)
    assert got["n_acc"].tolist() == n_acc
    assert got["tokens"].dtype == tokens.dtype and got["tokens"].tolist() == out
    assert got["path"].tolist() == path
    return n_acc


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("B,N,V", [(1, 1, 1), (1, 1, 1000), (3, 2, 2), (5, 7, 40), (4, 26, 1000), (2, 64, 1024), (3, 65, 1025), (1, 256, 300), (2, 20, 32000),
                                   (40, 12, 5000), (1, 8, 131072), (3, 9, 65537), (9, 30, 70001), (300, 5, 257)])
def test_sizes(dtype, wide, B, N, V):
    run(*inputs(B, N, V, dtype, wide=wide))


def test_trees_that_are_walked_far_down():
    # chains of certain tokens: all nodes are kept
    for N in (2, 30, 64, 65, 256):
        B, V = 3, 50
        parents = random_tree(B, N, 0, chain=True)
        tokens = (torch.arange(B)[:, None] * 7 + torch.arange(N)) % V
        p = torch.zeros(B, N, V)
        p[:, : N - 1].scatter_(2, tokens[:, 1:, None], 1.0)
        p[:, N - 1, 3] = 1.0
        n_acc = run(tokens.to(torch.int32).cuda(), parents.cuda(), p.cuda(), torch.rand(B, N, generator=torch.Generator().manual_seed(1)).cuda())
        assert n_acc == [N - 1] * B


def test_one_tree_for_all():
    tokens, parents, p, u = inputs(6, 20, 300)
    run(tokens, parents[0].contiguous(), p, u)


@pytest.mark.parametrize("V", [100, 66000])
def test_ragged_and_empty(V):
    tokens, parents, p, u = inputs(7, 15, V, sharp=8.0)
    n_new = torch.tensor([0, 1, 2, 15, 99, -4, 8], dtype=torch.int32).cuda()
    n_acc = run(tokens, parents, p, u, n_new=n_new)
    assert n_acc[0] == n_acc[5] == -1
    run(tokens, parents, choices=p.argmax(-1).to(torch.int32), n_new=n_new)


@pytest.mark.parametrize("V", [50, 66000])
def test_trees_that_are_none(V):
    # entries that name no earlier node, several nodes of one token, tokens outside the vocabulary
    tokens, parents, p, u = inputs(8, 30, V, sharp=6.0)
    parents[0, 5:], parents[1, 7], parents[2, 3], parents[3] = -1, 7, 29, 0
    parents[4, 0], parents[5, 0], parents[6, 9] = 3, 2 ** 31 - 1, -2 ** 31
    tokens[3] = tokens[3, 1]
    tokens[4, ::2], tokens[5, ::3], tokens[6, 4] = -1, V, 2 ** 31 - 1
    run(tokens, parents, p, u)


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("V", [400, 3472, 66000])
def test_weights_that_are_none(dtype, V):
    # at every place of a load
    tokens, parents, p, u = inputs(16, 4, V, dtype)
    for b in range(16):
        p[b, 0, b], p[b, 1:, V - 1 - b] = (math.inf, math.nan, -2.0, -math.inf)[b % 4], math.inf
    run(tokens, parents, p, u)
    tokens, parents, p, u = inputs(6, 10, V, dtype)
    p[0], p[1, 0], p[2, 0, 7], p[3, 0, 5], p[4, :, 100:] = 0.0, -0.5, math.nan, math.inf, 0.0
    tokens[0] = -1                                             # a draw of -1 is no node's token
    run(tokens, parents, p, u)
    u[:] = 1 - 2 ** -24                                        # the largest below 1, and 0
    run(tokens, parents, p, u)
    u[:] = 0.0
    run(tokens, parents, p, u)


def test_choices():
    for wide in (False, True):
        tokens, parents, p, u = inputs(9, 40, 60, sharp=6.0, wide=wide)
        choices = p.argmax(-1).to(tokens.dtype)
        assert max(run(tokens, parents, choices=choices)) > 1
        choices[0, 0], choices[1] = -7, 2 ** 31 - 1
        run(tokens, parents, choices=choices)


def test_strides():
    tokens, parents, p, u = inputs(4, 9, 301)
    wide = torch.zeros(4, 12, 310).cuda()
    wide[:, 2:11, 5:306] = p
    run(tokens, parents, wide[:, 2:11, 5:306], u)              # rows that start anywhere
    run(tokens, parents, p.transpose(0, 1).contiguous().transpose(0, 1), u)
    run(tokens, parents, p[:, :1].expand(4, 9, 301), u)


def test_kept_tokens_follow_the_targets_distribution():
    # the first token of 40000 rounds over one tree: counts within five standard deviations of what p says
    V, N, B = 8, 4, 40000
    p = torch.softmax(torch.randn(1, N, V, generator=torch.Generator().manual_seed(4)), -1)
    tokens = torch.tensor([0, 2, 5, 1], dtype=torch.int32).expand(B, N).contiguous().cuda()
    parents = torch.tensor([-1, 0, 0, 1], dtype=torch.int32).cuda()
    u = torch.rand(B, N, generator=torch.Generator().manual_seed(5)).cuda()
    got = tsd.verify_tree_static(tokens, parents, p=p.expand(B, N, V).cuda(), uniforms=u)
    counts = torch.bincount(got["tokens"][:, 0].long(), minlength=V).double().cpu()
    want = p[0, 0].double()
    assert bool(((counts - B * want).abs() <= 5 * (B * want * (1 - want)).sqrt()).all())


@pytest.mark.parametrize("B,N,V", [(1, 26, 32000), (40, 12, 5000), (2, 12, 70000)])
def test_streams_and_replayed_graphs(B, N, V):
    tokens, parents, p, u = inputs(B, N, V)
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                got = tsd.verify_tree_static(tokens, parents, p=p, uniforms=u)
            graphs.append((g, got))
    torch.cuda.synchronize()
    for step in range(6):
        u.uniform_()
        torch.cuda.synchronize()
        want = tsd.verify_tree_static(tokens, parents, p=p, uniforms=u)
        for s, (g, got) in zip(streams, graphs):
            for x in got.values():
                x.fill_(-9)
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for _, got in graphs:
            assert all(torch.equal(want[k], got[k]) for k in want)
    n_acc, out, path = walked(tokens, parents, p, u)
    assert want["n_acc"].tolist() == n_acc and want["tokens"].tolist() == out and want["path"].tolist() == path


def test_offsets_beyond_32_bits():
    N, V = 200, 1 << 21
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs some 40 GB of device memory")
    B = 11                                                     # elements past 2^32
    p = torch.zeros(B, N, V, dtype=torch.bfloat16, device="cuda")
    tokens = torch.zeros(B, N, dtype=torch.int32)
    parents = torch.full((N,), -1, dtype=torch.int32)
    parents[N - 1] = 0
    for b in range(B):
        tokens[b, N - 1] = 17 * b + 3
        p[b, 0, 17 * b + 3], p[b, N - 1, V - 1 - b] = 1.0, 1.0
    got = tsd.verify_tree_static(tokens.cuda(), parents.cuda(), p=p, uniforms=torch.rand(B, N).cuda())
    assert got["n_acc"].tolist() == [1] * B
    assert got["tokens"][:, :3].tolist() == [[17 * b + 3, V - 1 - b, -1] for b in range(B)]
    assert got["path"][:, :3].tolist() == [[0, N - 1, -1]] * B
