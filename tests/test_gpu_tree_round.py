"""The calls together, as a program uses them: decoding of a small token model by trees of drafts, over the paged caches of all its layers in one pool.  The tree's
nodes are the draft's likeliest tokens; every committed token is checked against a forward pass over the whole history in 64 bits."""
import pytest
import torch

import paper_2511_18191_amd as tsd
from test_gpu_caller_round import BASE, HD, HKV, HQ, LAYERS, PAGE, V, Model, norm
from tree_ref import ALL, lines

pytestmark = pytest.mark.gpu


def forward(model, tokens, window, sinks):
    """Logits of a whole sequence, no cache, in the model's type on the host."""
    x, n = model.embed[tokens], len(tokens)
    freq = BASE ** (-torch.arange(0, HD, 2, dtype=torch.float64) / HD)
    angle = torch.arange(n)[:, None] * freq
    c, s = angle.cos()[:, None], angle.sin()[:, None]

    def turned(y):
        a, b = y[..., : HD // 2], y[..., HD // 2:]
        return torch.cat([a * c - b * s, a * s + b * c], -1)

    i, j = torch.arange(n)[:, None], torch.arange(n)[None]
    hidden = (j > i) | ((j <= i - window) & (j >= sinks))
    for layer in model.layers:
        q, k, v = (norm(x) @ layer["qkv"]).view(n, HQ + 2 * HKV, HD).split([HQ, HKV, HKV], 1)
        q, k, v = turned(q), turned(k).repeat_interleave(HQ // HKV, 1), v.repeat_interleave(HQ // HKV, 1)
        w = torch.softmax((torch.einsum("qhd,khd->hqk", q, k) / HD ** 0.5).masked_fill(hidden, -torch.inf), -1)
        x = x + torch.einsum("hqk,khd->qhd", w, v).flatten(1) @ layer["o"]
        x = x + torch.relu(norm(x) @ layer["up"]) @ layer["down"]
    return norm(x) @ model.head


class Cached:
    """The target on the GPU: all layers' caches in one pool [layers, pages, page, heads, dim]."""

    def __init__(self, model, B, most, window, sinks):
        self.m, cols = model, -(-most // PAGE)
        self.table = torch.randperm(B * cols, generator=torch.Generator().manual_seed(9)).to(torch.int32).view(B, cols).cuda()
        self.k, self.v = (torch.full((LAYERS, B * cols, PAGE, HKV, HD), float("nan"), device="cuda") for _ in range(2))
        self.freq, _ = tsd.rope_frequencies(HD, BASE)
        self.window, self.sinks = window, sinks

    def logits(self, tokens, held, n_new, parents=None, depth=None):
        x = self.m.embed[tokens]
        positions = None if depth is None else (held[:, None] + depth).to(torch.int32)
        for layer, k_pool, v_pool in zip(self.m.layers, self.k, self.v):
            q, k, v = (norm(x) @ layer["qkv"]).view(*tokens.shape, HQ + 2 * HKV, HD).split([HQ, HKV, HKV], 2)
            q = tsd.rope_append_static(q, k, v, k_pool, v_pool, self.table, held, self.freq, positions=positions, n_new=n_new,
                                       out=torch.zeros_like(q, memory_format=torch.contiguous_format))
            if parents is not None:
                a = tsd.tree_attn_static(q, k_pool, v_pool, self.table, held + n_new, parents, window=self.window if self.window < ALL else None,
                                         sinks=self.sinks, n_new=n_new, out=torch.zeros_like(q))
            else:
                a = tsd.window_attn_static(q, k_pool, v_pool, self.table, held + n_new, self.window, sinks=self.sinks, n_new=n_new, out=torch.zeros_like(q))
            x = x + a.flatten(2) @ layer["o"]
            x = x + torch.relu(norm(x) @ layer["up"]) @ layer["down"]
        return norm(x) @ self.m.head


@pytest.mark.parametrize("greedy,window,sinks", [(True, ALL, 0), (False, ALL, 0), (False, 12, 2), (True, 5, 0)])
def test_decoding_by_trees(greedy, window, sinks):
    B, length, most, wide = 4, 45, 112, (3, 2, 1)               # three children of the root, two of each of those, one of each of those
    parents, depth = [-1], [0]
    for level, children in enumerate(wide):
        for n in [i for i, d in enumerate(depth) if d == level]:
            parents += [n] * children
            depth += [level + 1] * children
    N = len(parents)
    assert lines(parents, N)[0].tolist() == depth
    target = Model(LAYERS, 1).to("cuda", torch.float32)
    draft = Model(LAYERS, 1).to("cpu", torch.float64)
    draft.layers = draft.layers[:1]                              # the draft leaves out the target's last layer
    T, g = Cached(target, B, most, window, sinks), torch.Generator().manual_seed(3)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    history = [torch.randint(0, V, (n,), generator=g).tolist() for n in (3, 17, 9, 30)]
    padded = torch.zeros(B, 30, dtype=torch.long)
    for b, h in enumerate(history):
        padded[b, : len(h) - 1] = torch.tensor(h[:-1])
    T.logits(padded.cuda(), i32([0] * B), i32([len(h) - 1 for h in history]))
    held = [len(h) - 1 for h in history]
    tree, deep = i32(parents), torch.tensor(depth).cuda()
    checks, kept_nodes = [], 0
    while min(len(h) for h in history) < length:
        live = [len(h) < length for h in history]
        nodes = torch.zeros(B, N, dtype=torch.int32)
        nodes[:, 0] = torch.tensor([h[-1] for h in history])
        for level, children in enumerate(wide):                  # a level at a time: the likeliest tokens behind every node of the one above
            above = [i for i, d in enumerate(depth) if d == level]
            rows = []
            for b, h in enumerate(history):
                for n in above:
                    way = []
                    while n > 0:
                        way.insert(0, int(nodes[b, n]))
                        n = parents[n]
                    rows.append(forward(draft, torch.tensor(h + way), window, sinks)[-1])
            ids = tsd.token_logprobs_static(torch.stack(rows).view(B, len(above), V).float().cuda(), top=children)["top_ids"].cpu()
            for i, n in enumerate(above):
                for c in [c for c in range(N) if parents[c] == n]:
                    nodes[:, c] = ids[:, i, c - min(c for c in range(N) if parents[c] == n)]
        n_new = i32([N if x else 0 for x in live])
        base = i32(held)
        logits = T.logits(nodes.cuda(), base, n_new, tree, deep)
        if greedy:
            got = tsd.verify_tree_static(nodes.cuda(), tree, choices=tsd.token_logprobs_static(logits, top=1, n_new=n_new)["top_ids"][..., 0].contiguous(), n_new=n_new)
        else:
            got = tsd.verify_tree_static(nodes.cuda(), tree, p=torch.softmax(logits, -1), uniforms=torch.rand(B, N, generator=g).cuda(), n_new=n_new)
        tsd.keep_path_static(T.k, T.v, T.table, base, got["path"])
        n_acc, out, path = got["n_acc"].tolist(), got["tokens"].tolist(), got["path"].tolist()
        for b, h in enumerate(history):
            if not live[b]:
                assert n_acc[b] == -1 and set(out[b] + path[b]) == {-1}
                continue
            new = out[b][: n_acc[b] + 1]
            assert all(0 <= t < V for t in new) and [int(nodes[b, n]) for n in path[b][1: n_acc[b] + 1]] == new[:-1]
            checks.append((b, len(h), logits[b, path[b][: n_acc[b] + 1]].cpu()))
            held[b] += n_acc[b] + 1
            h.extend(new)
            kept_nodes += n_acc[b]
            assert held[b] == len(h) - 1
    assert kept_nodes > 0
    exact = Model(LAYERS, 1).to("cpu", torch.float64)
    want = [forward(exact, torch.tensor(h), window, sinks) for h in history]
    for b, start, x in checks:
        for i in range(len(x)):
            at = want[b][start + i - 1]
            # (fp32, two layers: 1e-4 of logits of 3, as where chains are drafted)
            assert torch.allclose(torch.softmax(x[i].double(), -1), torch.softmax(at, -1), atol=1e-4)
            if greedy:
                assert float(at.max() - at[history[b][start + i]]) < 1e-3
