"""The calls together, as a program uses them: speculative decoding of a small token transformer over paged caches.  Every committed token is
checked against a forward pass over the whole history in 64 bits."""
import pytest
import torch

import paper_2511_18191_amd as tsd

pytestmark = pytest.mark.gpu

V, WIDTH, HQ, HKV, HD, LAYERS, PAGE, BASE = 40, 64, 4, 2, 16, 2, 16, 10000.0


class Model:
    """Embedding, layers of attention and a two-matrix FFN, and a head; weights fixed by the seed."""

    def __init__(self, layers, seed):
        g = torch.Generator().manual_seed(seed)
        m = lambda *s: torch.randn(*s, generator=g) / s[0] ** 0.5
        self.embed, self.head = torch.randn(V, WIDTH, generator=g), 3 * m(WIDTH, V)
        self.layers = [dict(qkv=m(WIDTH, (HQ + 2 * HKV) * HD), o=m(HQ * HD, WIDTH), up=m(WIDTH, 2 * WIDTH), down=m(2 * WIDTH, WIDTH)) for _ in range(layers)]

    def to(self, device, dtype):
        self.embed, self.head = self.embed.to(device, dtype), self.head.to(device, dtype)
        self.layers = [{k: x.to(device, dtype) for k, x in layer.items()} for layer in self.layers]
        return self


def norm(x):
    return x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()


class Cached:
    """The model on the GPU over paged caches, its new tokens through the calls under test."""

    def __init__(self, model, B, most, interleaved):
        self.m, cols = model, -(-most // PAGE)
        g = torch.Generator().manual_seed(9)
        self.table = torch.randperm(B * cols, generator=g).to(torch.int32).view(B, cols).cuda()
        self.pools = [[torch.full((B * cols, PAGE, HKV, HD), float("nan"), device="cuda") for _ in range(2)] for _ in model.layers]
        self.freq, self.amplitude = tsd.rope_frequencies(HD, BASE, "linear", 2.0)
        self.interleaved = interleaved

    def logits(self, tokens, held, n_new):
        x = self.m.embed[tokens]
        for layer, (k_pool, v_pool) in zip(self.m.layers, self.pools):
            q, k, v = (norm(x) @ layer["qkv"]).view(*tokens.shape, HQ + 2 * HKV, HD).split([HQ, HKV, HKV], 2)
            q = tsd.rope_append_static(q, k, v, k_pool, v_pool, self.table, held, self.freq, n_new=n_new, interleaved=self.interleaved,
                                       amplitude=self.amplitude, out=torch.zeros_like(q, memory_format=torch.contiguous_format))
            a = tsd.paged_attn_static(q, k_pool, v_pool, self.table, held + n_new, n_new=n_new, out=torch.zeros_like(q))
            x = x + a.flatten(2) @ layer["o"]
            x = x + torch.relu(norm(x) @ layer["up"]) @ layer["down"]
        return norm(x) @ self.m.head


def reference(model, tokens, interleaved):
    """Logits of a whole sequence, no cache, in 64 bits."""
    x, n = model.embed[tokens], len(tokens)
    freq = BASE ** (-torch.arange(0, HD, 2, dtype=torch.float64) / HD) / 2.0
    turn = torch.polar(torch.ones(n, HD // 2, dtype=torch.float64), torch.arange(n)[:, None] * freq)[:, None]

    def turned(y):
        if interleaved:
            return torch.view_as_real(torch.view_as_complex(y.reshape(*y.shape[:-1], HD // 2, 2).contiguous()) * turn).flatten(-2)
        z = torch.complex(y[..., : HD // 2], y[..., HD // 2:]) * turn
        return torch.cat([z.real, z.imag], -1)

    for layer in model.layers:
        q, k, v = (norm(x) @ layer["qkv"]).view(n, HQ + 2 * HKV, HD).split([HQ, HKV, HKV], 1)
        q, k, v = turned(q), turned(k).repeat_interleave(HQ // HKV, 1), v.repeat_interleave(HQ // HKV, 1)
        s = torch.einsum("qhd,khd->hqk", q, k) / HD ** 0.5
        s = s.masked_fill(torch.ones(n, n).triu(1).bool(), -torch.inf)
        x = x + torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), v).flatten(1) @ layer["o"]
        x = x + torch.relu(norm(x) @ layer["up"]) @ layer["down"]
    return norm(x) @ model.head


@pytest.mark.parametrize("greedy,interleaved", [(True, False), (False, True)])
def test_speculative_decoding_of_a_token_model(greedy, interleaved):
    B, K, length, most = 5, 4, 60, 128
    target, draft = Model(LAYERS, 1).to("cuda", torch.float32), Model(LAYERS, 1).to("cuda", torch.float32)
    draft.layers = draft.layers[:1]                              # the draft leaves out the target's last layer
    T, D = Cached(target, B, most, interleaved), Cached(draft, B, most, interleaved)
    torch.manual_seed(5)
    g = torch.Generator().manual_seed(3)
    prompt_len = [3, 17, 9, 1, 30]
    history = [torch.randint(0, V, (n,), generator=g).tolist() for n in prompt_len]
    probabilities = (lambda x: torch.nn.functional.one_hot(x.argmax(-1), V).float()) if greedy else (lambda x: torch.softmax(x, -1))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    for C in (T, D):                                             # prompts but their last token, as one padded batch
        padded = torch.zeros(B, 30, dtype=torch.long)
        for b, h in enumerate(history):
            padded[b, : len(h) - 1] = torch.tensor(h[:-1])
        C.logits(padded.cuda(), i32([0] * B), i32([len(h) - 1 for h in history]))
    in_target, in_draft, passed = [len(h) - 1 for h in history], [len(h) - 1 for h in history], 0
    checks = []
    while min(len(h) for h in history) < length:
        ask = [0 if len(h) >= length else min(K, 1 + b) for b, h in enumerate(history)]     # ragged drafts; finished sequences ask for none
        drafts, qs = torch.zeros(B, K, dtype=torch.long).cuda(), torch.zeros(B, K, V).cuda()
        for i in range(K):                                       # the draft takes what it has not seen, one or two tokens, then its own
            feed = [h[n:] for h, n in zip(history, in_draft)] if i == 0 else [[int(drafts[b, i - 1])] for b in range(B)]
            width = max(len(f) for f in feed)
            tokens = torch.tensor([f + [0] * (width - len(f)) for f in feed]).cuda()
            held = in_draft if i == 0 else [len(h) + i - 1 for h in history]
            out = D.logits(tokens, i32(held), i32([len(f) for f in feed]))
            qs[:, i] = probabilities(out[torch.arange(B), [len(f) - 1 for f in feed]])
            drafts[:, i] = torch.multinomial(qs[:, i], 1)[:, 0]
        tokens = torch.cat([torch.tensor([h[-1:] for h in history]).cuda(), drafts], 1)
        p = probabilities(T.logits(tokens, i32(in_target), i32([a + 1 for a in ask])))
        got = tsd.verify_tokens_static(drafts, qs, p, torch.rand(B, K + 1, generator=g).cuda(), n_draft=i32(ask))
        counts, out = got["n_acc"].tolist(), got["tokens"].tolist()
        for b, h in enumerate(history):
            if len(h) >= length:
                continue
            assert 0 <= counts[b] <= ask[b] and out[b][counts[b] + 1:] == [-1] * (K - counts[b])
            new = out[b][: counts[b] + 1]
            assert all(0 <= t < V for t in new)
            checks.append((b, len(h), p[b, : len(new)].cpu()))
            in_target[b] = len(h) + counts[b]                    # rolled back by holding fewer
            in_draft[b] = min(len(h) + counts[b], len(h) + K - 1)
            h.extend(new)
            passed += counts[b]
    assert passed > 0
    exact = Model(LAYERS, 1).to("cpu", torch.float64)
    logits = [reference(exact, torch.tensor(h), interleaved) for h in history]
    for b, start, p in checks:
        for i in range(len(p)):
            at = logits[b][start + i - 1]
            if greedy:
                # the token itself: the largest logit, or one that rounding cannot tell from it (fp32, two layers: 1e-4 of logits of 3)
                assert float(at.max() - at[history[b][start + i]]) < 1e-3
            else:
                assert torch.allclose(p[i].double(), torch.softmax(at, -1), atol=1e-4)
